// qgemm_tokens.hip -- the quantized linear layer with a step per token where there are few tokens: a decode step's.
//
// Its weights are read once and meet at most 64 rows, so that the weights' bytes bound it.  As in qgemm_skinny.hip there are
// no LDS tiles: both operands are K-contiguous, the operand layout of v_mfma_i32_16x16x64_i8, and a lane loads its operands
// straight into registers; the waves of a workgroup deal the k steps out between them and their accumulators meet in LDS
// (integers: exact in any order).  A k step is 128 bytes of a weight row, a whole cache line: 128 k of int8 weights, 256 of
// packed ones.  A workgroup takes NT x 16 output channels and all rows (MT x 16), which come out of the L2.
// 8 x 4096 x 8192 read 33.6 MB of weights in 10.3 us (3.3 TB/s), 64 x 4096 x 4096 in 13.7 us: from 33 rows on the rows, which
// every workgroup reads out of the L2, bound it (with rows of zero bytes 7.6 us).
//
// With few values in at most 16 rows the rows' quantizer (token_quant.hip's arithmetic, bit for bit) runs in the same kernel: each
// workgroup takes the rows' maxima itself, a wave a row, while its weights are on their way, and quantizes the values
// of its k steps as it loads them.  That spares a launch (3.9 us of host time) and a kernel's latency.
#include "qgemm_dma.hpp"

namespace mpq {

constexpr int kTokWaves = 8, kTokThreads = kTokWaves * 64;

struct TokArgs {
  const void* a;       // codes int8 [M x K], or the rows themselves, a_stride elements apart
  const void* w;
  int64_t a_stride;
  int M, K;
  int64_t N;
  const float* a_scale;
  const float* w_scale;
  int w_per_row, act, y_type, bits;
  void* y;
};

// 16 codes of a row's 16 values
template <int SRC>
__device__ __forceinline__ v4i quantize16(const typename Elem<SRC>::type* x, float inv) {
  const f32x8 a = Elem<SRC>::load8(x), b = Elem<SRC>::load8(x + 8);
  float t[16];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t[e] = __builtin_fmaf(a[e], inv, kMagic);
    t[8 + e] = __builtin_fmaf(b[e], inv, kMagic);
  }
  return v4i{(int)low_bytes(t[0], t[1], t[2], t[3]), (int)low_bytes(t[4], t[5], t[6], t[7]),
             (int)low_bytes(t[8], t[9], t[10], t[11]), (int)low_bytes(t[12], t[13], t[14], t[15])};
}

// SRC: type of the rows that are quantized here (MT 1, K % 16 == 0), or -1: codes.  Rows of at least 16 bytes.
template <int MT, int NT, bool W4, int SRC>
__global__ __launch_bounds__(kTokThreads, 2) void token_rows_k(TokArgs p) {
  constexpr int NW = kTokWaves, KSTEP = W4 ? 256 : 128;
  constexpr int HALF = W4 ? 2 : 1;  // operands that a 16-byte chunk of weights makes
  constexpr bool FUSED = SRC >= 0;
  typedef typename Elem<FUSED ? SRC : MPQ_F32>::type El;
  __shared__ v4i red[NW][MT * NT][64];
  __shared__ float row_max[FUSED ? 16 : 1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, q = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
  const int K = p.K, w_bytes = W4 ? K >> 1 : K;
  // rows past the edge re-read the last row; never stored
  const char* w_base = reinterpret_cast<const char*>(p.w) + n0 * w_bytes;
  unsigned w_row[NT], a_row[MT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t left = p.N - 1 - n0;
    const int n = j * 16 + r;
    w_row[j] = (unsigned)(n < left ? n : (int)left) * (unsigned)w_bytes;
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = i * 16 + r;
    a_row[i] = (unsigned)(m < p.M ? m : p.M - 1) * (unsigned)K;
  }
  const El* x_row = reinterpret_cast<const El*>(p.a) + (int64_t)(r < p.M ? r : p.M - 1) * p.a_stride;

  const int steps = (K + KSTEP - 1) / KSTEP;
  // One step's operands at a time: other waves hide a wave's wait better than further loads of its own (us with 1 | 2 | 4 steps
  // in flight, in a graph, weights from memory: 8 x 4096 x 8192 10.3 | 11.6 | 11.5, 19 x 4096 x 12288 packed 10.1 | 11.1 | 18.8,
  // 64 x 4096 x 4096 13.7 | 14.3 | 14.3).
  v4i w[NT][2], a[MT][2 * HALF];
  // k of the lane's weight chunk c of step s; chunks that would pass the row's end are loaded so that they end there
  auto k_of = [&](int s, int c) { return s * KSTEP + (W4 ? c * 128 + q * 32 : c * 64 + q * 16); };
  auto load_w = [&](int s) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int at = W4 ? k_of(s, c) >> 1 : k_of(s, c);
      const unsigned off = (unsigned)(at < w_bytes - 16 ? at : w_bytes - 16);
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j][c] = *reinterpret_cast<const v4i_byte*>(w_base + (w_row[j] + off));
    }
  };
  float inv = 0.0f, step = 0.0f;
  auto load_a = [&](int s) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int h = 0; h < HALF; ++h) {
        const int at = k_of(s, c) + 16 * h;
        const unsigned off = (unsigned)(at < K - 16 ? at : K - 16);
        if constexpr (FUSED) {
          a[0][c * HALF + h] = quantize16<SRC>(x_row + off, inv);
        } else {
#pragma unroll
          for (int i = 0; i < MT; ++i)
            a[i][c * HALF + h] = *reinterpret_cast<const v4i_byte*>(reinterpret_cast<const char*>(p.a) + (a_row[i] + off));
        }
      }
  };
  v4i acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4i{0, 0, 0, 0};
  if (wave < steps) load_w(wave);
  if constexpr (FUSED) {
    for (int m = wave; m < p.M; m += NW) {  // a wave a row
      const El* x = reinterpret_cast<const El*>(p.a) + m * p.a_stride;
      float top = 0.0f;
#pragma unroll 4
      for (int k = lane * 8; k < K; k += 512) {
        const f32x8 v = Elem<SRC>::load8(x + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
      }
      top = wave_max(top);
      if (lane == 0) row_max[m] = top;
    }
    __syncthreads();
    step_constants(row_max[r < p.M ? r : p.M - 1], p.bits, step, inv);
  }
  for (int s = wave; s < steps; s += NW) {
    if (s != wave) load_w(s);
    load_a(s);
    if ((s + 1) * KSTEP > K) {  // the step that reaches past the rows' end
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int j = 0; j < NT; ++j) w[j][c] = fix_chunk16(w[j][c], w_bytes, W4 ? k_of(s, c) >> 1 : k_of(s, c));
        if (!FUSED) {  // (a chunk of values lies within the row, or wholly behind it, next to weights of zero)
#pragma unroll
          for (int h = 0; h < HALF; ++h)
#pragma unroll
            for (int i = 0; i < MT; ++i) a[i][c * HALF + h] = fix_chunk16(a[i][c * HALF + h], K, k_of(s, c) + 16 * h);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        v4i b[HALF];
        if constexpr (W4) {  // 32 nibbles -> 32 bytes n << 4, in k order
          unsigned e[8];
#pragma unroll
          for (int d = 0; d < 4; ++d) expand8((unsigned)w[j][c][d], e[2 * d], e[2 * d + 1]);
          b[0] = v4i{(int)e[0], (int)e[1], (int)e[2], (int)e[3]};
          b[HALF - 1] = v4i{(int)e[4], (int)e[5], (int)e[6], (int)e[7]};
        } else {
          b[0] = w[j][c];
        }
#pragma unroll
        for (int h = 0; h < HALF; ++h)
#pragma unroll
          for (int i = 0; i < MT; ++i)  // W as the row operand: a lane then holds four consecutive n of one output row
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[h], a[i][c * HALF + h], acc[i][j], 0, 0, 0);
      }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) red[wave][i * NT + j][lane] = acc[i][j];
  __syncthreads();
  // the waves share out the accumulator tiles
  for (int t = wave; t < MT * NT; t += NW) {
    v4i sum = red[0][t][lane];
#pragma unroll
    for (int v = 1; v < NW; ++v) sum += red[v][t][lane];
    const int m = (t / NT) * 16 + r;
    const int64_t n = n0 + (t % NT) * 16 + 4 * q;
    if (m >= p.M || n >= p.N) continue;
    const float sa = FUSED ? step : p.a_scale[m];
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int v = W4 ? sum[e] >> 4 : sum[e];  // exact: every product carried the factor 16
      const float sw = p.w_scale[p.w_per_row ? (n + e < p.N ? n + e : n) : 0];
      y[e] = apply_act(((float)v * sa) * sw, p.act);
    }
    const bool whole = n + 4 <= p.N;
    if (p.y_type == MPQ_F32) {
      float* out = reinterpret_cast<float*>(p.y) + m * p.N + n;
      if (whole) store4(out, make_float4(y[0], y[1], y[2], y[3]));
      else
        for (int e = 0; e < 4 && n + e < p.N; ++e) out[e] = y[e];
    } else {
      unsigned short* out = reinterpret_cast<unsigned short*>(p.y) + m * p.N + n;
      const v2i h = to_half4(make_float4(y[0], y[1], y[2], y[3]), p.y_type == MPQ_BF16);
      if (whole) *reinterpret_cast<v2i_any*>(out) = h;
      else
        for (int e = 0; e < 4 && n + e < p.N; ++e) out[e] = (unsigned short)((unsigned)(e < 2 ? h.x : h.y) >> (16 * (e & 1)));
    }
  }
}

// (a grid counts 2^32 threads)
bool token_rows(bool w4, int64_t M, int64_t N, int64_t K) { return M <= 64 && N <= (1 << 26) && K >= (w4 ? 32 : 16); }
// Every workgroup reads and quantizes all rows, so that there must not be much of them (us on the device, one kernel | two;
// a launch more costs the host 4: 1 x 4096 x 4096 6.8 | -, 8 x 4096 x 4096 packed 7.9 | 8.8, 16 x 4096 x 4096 11.9 | 10.7, x 12288 fp32
// 23.1 | 17.9, 16 x 11008 x 4096 27.1 | 21.1; with more than 16 rows 32 x 1024 x 1024 8.3 | 6.5, 19 x 4096 x 12288 packed 24.6 | 13.8).
bool token_rows_fused(bool w4, int64_t M, int64_t N, int64_t K) {
  return token_rows(w4, M, N, K) && M <= 16 && K % 16 == 0 && M * K <= 65536;
}

// Channel tiles per workgroup: what makes the bytes that a CU loads smallest, its workgroups' weights and rows.
static int channel_tiles(int mt, bool w4, const TokArgs& p, int el) {
  int best = 1;
  double least = 0;
  for (int nt = 1; nt <= (mt == 4 ? 2 : 4); ++nt) {
    const int64_t groups = (p.N + 16 * nt - 1) / (16 * nt), rounds = (groups + kNumCU - 1) / kNumCU;
    const double bytes = (double)rounds * (nt * 16 * (w4 ? 0.5 : 1.0) + mt * 16 * el);
    if (nt == 1 || bytes < least) { least = bytes; best = nt; }
  }
  return best;
}

template <int MT, bool W4, int SRC>
static int go(const TokArgs& p, hipStream_t st) {
  const int nt = channel_tiles(MT, W4, p, SRC < 0 ? 1 : SRC == MPQ_F32 ? 4 : 2);
  const unsigned grid = (unsigned)((p.N + 16 * nt - 1) / (16 * nt));
  if (nt == 1) token_rows_k<MT, 1, W4, SRC><<<grid, kTokThreads, 0, st>>>(p);
  else if (nt == 2) token_rows_k<MT, 2, W4, SRC><<<grid, kTokThreads, 0, st>>>(p);
  if constexpr (MT < 4) {
    if (nt == 3) token_rows_k<MT, 3, W4, SRC><<<grid, kTokThreads, 0, st>>>(p);
    else if (nt == 4) token_rows_k<MT, 4, W4, SRC><<<grid, kTokThreads, 0, st>>>(p);
  }
  return launch_status();
}

int launch_token_rows(bool w4, const DmaArgs& d) {
  const TokArgs p{d.a_q, d.w_q, d.K, (int)d.M, (int)d.K, d.N, d.a_scale, d.w_scale, d.per_row, d.epi.act, d.epi.y_type, 8, d.y_out};
  if (d.M <= 16) return w4 ? go<1, true, -1>(p, d.st) : go<1, false, -1>(p, d.st);
  if (d.M <= 32) return w4 ? go<2, true, -1>(p, d.st) : go<2, false, -1>(p, d.st);
  return w4 ? go<4, true, -1>(p, d.st) : go<4, false, -1>(p, d.st);
}

int launch_token_rows_fused(const void* x, int x_type, int64_t x_stride, int bits, bool w4, const DmaArgs& d) {
  const TokArgs p{x, d.w_q, x_stride, (int)d.M, (int)d.K, d.N, nullptr, d.w_scale, d.per_row, d.epi.act, d.epi.y_type, bits, d.y_out};
  if (x_type == MPQ_F32) return w4 ? go<1, true, MPQ_F32>(p, d.st) : go<1, false, MPQ_F32>(p, d.st);
  if (x_type == MPQ_BF16) return w4 ? go<1, true, MPQ_BF16>(p, d.st) : go<1, false, MPQ_BF16>(p, d.st);
  return w4 ? go<1, true, MPQ_F16>(p, d.st) : go<1, false, MPQ_F16>(p, d.st);
}

}  // namespace mpq
