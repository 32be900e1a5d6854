// qgemm_tokens.hip -- the quantized linear layer with a step per token where there are few tokens: a decode step's.
//
// Its weights are read once and meet at most 64 rows, so that the weights' bytes bound it.  As in qgemm_skinny.hip there are
// no LDS tiles: both operands are K-contiguous, the operand layout of v_mfma_i32_16x16x64_i8, and a lane loads its operands
// straight into registers; the waves of a workgroup deal the k steps of 128 out between them and their accumulators
// meet in LDS (integers: exact in any order).  A workgroup takes NT x 16 output channels and all rows (MT x 16), which come
// out of the L2: rows are read once per NT x 16 channels.
#include "qgemm_dma.hpp"

namespace mpq {

constexpr int kTokWaves = 8;

template <int MT, int NT, bool W4>
__global__ __launch_bounds__(kTokWaves * 64) void token_skinny_k(const int8_t* __restrict__ A, const void* __restrict__ Wv, int64_t M,
                                                                 int64_t N, int64_t K, const float* __restrict__ a_scale,
                                                                 const float* __restrict__ w_scale, int w_per_row,
                                                                 void* __restrict__ Y, int act, int y_type) {
  constexpr int NW = kTokWaves;
  constexpr int CB = W4 ? 1 : 2;  // 16-byte chunks of a W row per lane and step
  constexpr int QA = W4 ? 32 : 16, HA = W4 ? 16 : 64;  // see qgemm_skinny
  __shared__ v4i red[NW][MT * NT][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, q = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
  const int kb_a = (int)K, kb_w = W4 ? (int)(K >> 1) : (int)K;  // bytes per row
  const uint8_t* pa[MT];
  const uint8_t* pw[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {  // rows past the edge re-read the last row; never stored
    const int64_t m = i * 16 + r;
    pa[i] = reinterpret_cast<const uint8_t*>(A) + (m < M ? m : M - 1) * kb_a;
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t n = n0 + j * 16 + r;
    pw[j] = reinterpret_cast<const uint8_t*>(Wv) + (n < N ? n : N - 1) * kb_w;
  }
  v4i acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4i{0, 0, 0, 0};

  const int steps = (int)((K + 127) >> 7);
  constexpr int U = MT * 2 + NT * CB <= 6 ? 4 : 2;  // k steps whose loads are in flight together
  for (int s0 = wave; s0 < steps; s0 += NW * U) {
    v4i a[U][MT][2], b[U][NT][CB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u * NW;
      if (s < steps) {  // wave-uniform
        const int ka = s * 128 + q * QA, kw = W4 ? ka >> 1 : ka;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int c = 0; c < CB; ++c) b[u][j][c] = load_chunk16(pw[j], kb_w, kw + HA * c);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          a[u][i][0] = load_chunk16(pa[i], kb_a, ka);
          a[u][i][1] = load_chunk16(pa[i], kb_a, ka + HA);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u * NW;
      if (s < steps) {
        const int ka = s * 128 + q * QA, kw = W4 ? ka >> 1 : ka;
        if (s == steps - 1) {  // the step that may reach past the row's end
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            a[u][i][0] = fix_chunk16(a[u][i][0], kb_a, ka);
            a[u][i][1] = fix_chunk16(a[u][i][1], kb_a, ka + HA);
          }
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int c = 0; c < CB; ++c) b[u][j][c] = fix_chunk16(b[u][j][c], kb_w, kw + HA * c);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          v4i bw[2] = {b[u][j][0], b[u][j][CB - 1]};
          if constexpr (W4) {  // 32 nibbles -> 32 bytes n << 4, in k order
            unsigned e[8];
            expand8((unsigned)b[u][j][0].x, e[0], e[1]);
            expand8((unsigned)b[u][j][0].y, e[2], e[3]);
            expand8((unsigned)b[u][j][0].z, e[4], e[5]);
            expand8((unsigned)b[u][j][0].w, e[6], e[7]);
            bw[0] = v4i{(int)e[0], (int)e[1], (int)e[2], (int)e[3]};
            bw[1] = v4i{(int)e[4], (int)e[5], (int)e[6], (int)e[7]};
          }
#pragma unroll
          for (int i = 0; i < MT; ++i) {  // W as the row operand: a lane then holds four consecutive n of one output row
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bw[0], a[u][i][0], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bw[1], a[u][i][1], acc[i][j], 0, 0, 0);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) red[wave][i * NT + j][lane] = acc[i][j];
  __syncthreads();
  // the waves share out the accumulator tiles
  for (int t = wave; t < MT * NT; t += NW) {
    v4i s = red[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) s += red[w][t][lane];
    const int64_t m = (t / NT) * 16 + r, n = n0 + (t % NT) * 16 + 4 * q;
    if (m >= M || n >= N) continue;
    const float sa = a_scale[m];
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int a = W4 ? s[e] >> 4 : s[e];  // exact: every product carried the factor 16
      const float sw = w_scale[w_per_row ? (n + e < N ? n + e : n) : 0];
      y[e] = apply_act(((float)a * sa) * sw, act);
    }
    const bool whole = n + 4 <= N;
    if (y_type == MPQ_F32) {
      float* out = reinterpret_cast<float*>(Y) + m * N + n;
      if (whole) store4(out, make_float4(y[0], y[1], y[2], y[3]));
      else
        for (int e = 0; e < 4 && n + e < N; ++e) out[e] = y[e];
    } else {
      unsigned short* out = reinterpret_cast<unsigned short*>(Y) + m * N + n;
      const v2i h = to_half4(make_float4(y[0], y[1], y[2], y[3]), y_type == MPQ_BF16);
      if (whole) *reinterpret_cast<v2i_any*>(out) = h;
      else
        for (int e = 0; e < 4 && n + e < N; ++e) out[e] = (unsigned short)((unsigned)(e < 2 ? h.x : h.y) >> (16 * (e & 1)));
    }
  }
}

bool token_skinny(int64_t M, int64_t N, int64_t K) { return M <= 64 && N <= (1 << 26); }  // (a grid counts 2^32 threads)

int launch_token_skinny(bool w4, const DmaArgs& d) {
  const int nt = d.N >= 32 * 128 ? 2 : 1;  // two channel tiles once that leaves half of the CUs one
  const unsigned grid = (unsigned)((d.N + 16 * nt - 1) / (16 * nt));
#define MPQ_TOK(MT_, NT_, W4_)                                                                                              \
  token_skinny_k<MT_, NT_, W4_><<<grid, kTokWaves * 64, 0, d.st>>>(d.a_q, d.w_q, d.M, d.N, d.K, d.a_scale, d.w_scale, d.per_row, \
                                                                   d.y_out, d.epi.act, d.epi.y_type)
#define MPQ_TOK_M(NT_, W4_) \
  (d.M <= 16 ? (void)MPQ_TOK(1, NT_, W4_) : d.M <= 32 ? (void)MPQ_TOK(2, NT_, W4_) : (void)MPQ_TOK(4, NT_, W4_))
  if (nt == 2) {
    if (w4) MPQ_TOK_M(2, true);
    else MPQ_TOK_M(2, false);
  } else {
    if (w4) MPQ_TOK_M(1, true);
    else MPQ_TOK_M(1, false);
  }
#undef MPQ_TOK_M
#undef MPQ_TOK
  return launch_status();
}

}  // namespace mpq
