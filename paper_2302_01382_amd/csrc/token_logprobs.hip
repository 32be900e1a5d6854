// token_logprobs.hip -- log probabilities of given tokens, entropy and the most probable alternatives, from one read of the logits.
//
// With m the row's largest logit, d = scale log2(e) (x - m), l = sum 2^d and w = sum d 2^d:
//   ln p_t = scale (x_t - m) - ln l,   entropy = ln l - ln 2 w / l.
// A scale below 1 is split into its power of two, unit, and a factor of 1 to 2: d = factor log2(e) (unit x - unit m), the difference in one fused
// step, so that logits further apart than fp32's range lose nothing, and no factor its bits, however small the scale is.
// A workgroup holds a piece of a row in registers, so that the maximum is known before the first exponential and nothing is
// rescaled in the loop.  The largest `top` of a piece: of the 64 maxima of what the threads of a lane number hold, the
// top-th largest is a bound that at least `top` values reach and few more do; those are listed, and a value's place in the order is
// the number of listed ones before it.  Where too many share the bound (all logits equal, say), they are taken one at a time.
// Rows of several pieces are joined by a workgroup each.
// Bytes and vector instructions bound it together where rows are many: 2500 x 65536 bf16, 328 MB, 62.7 us and 6.7 for the join, the vector ALUs
// busy for 78 % of it, a third of that with the exponentials; 190 x 100003 fp32, 76 MB, 17.3 and 4.0; a single row is latency, 5.8.
#include "types.hpp"

#include <cmath>

namespace mpq {

constexpr int kMostTop = 32, kPieceThreads = 256, kWideThreads = 1024, kListed = 1024;
constexpr int64_t kMostVocab = 1 << 22;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// 2^-200 is 0 in fp32: as the least exponent it leaves minus infinity a product of 0
constexpr float kLeast = -200.0f;

typedef unsigned long long Key;

struct Piece {
  float m, l, w;
};
struct LogprobArgs {
  const void* logits;
  int64_t rows, vocab, stride;
  float unit, factor;  // scale: their product; unit: a power of two, at most 1
  const int32_t* tokens;
  float* logprob;
  float* entropy;
  int top;
  float* top_logprob;
  int32_t* top_index;
  int pieces;
  Piece* piece;       // pieces > 1: [row][piece], then
  Key* best;          // [row][piece][top]
};

// A logit and its index as a number that is the larger the earlier it comes: by value, the lower index first where they are equal (-0
// and 0 are).  0 is none.
__device__ __forceinline__ unsigned order_of(float x) {
  const unsigned u = (unsigned)bits_from_f(x + 0.0f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned order) {
  return f_from_bits((int)(order & 0x80000000u ? order ^ 0x80000000u : ~order));
}
__device__ __forceinline__ Key key_of(float x, int index) { return (Key)order_of(x) << 32 | (unsigned)~index; }
__device__ __forceinline__ float value_of(Key k) { return value_of((unsigned)(k >> 32)); }
__device__ __forceinline__ int index_of(Key k) { return (int)~(unsigned)k; }

// An order that at least `top` of what 64 lanes hold reaches, from the lanes' largest: the upper half of the top-th largest, its bits from the
// highest down; at least that of the lowest number, so that minus infinity and none stay below.
__device__ __forceinline__ unsigned bound_of(unsigned largest, int top) {
  unsigned least = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const unsigned with = least | 1u << bit;
    least = __popcll(__ballot(largest >= with)) >= top ? with : least;
  }
  return max(least, 0x00800000u);
}

// The first `top` of n keys, in order, to out (those behind the last are 0): a key's place is the number of larger ones.  All threads;
// keys are there and out is cleared already.
template <int THREADS>
__device__ __forceinline__ void place_keys(const Key* keys, int n, int top, Key* out) {
  for (int k = threadIdx.x; k < n; k += THREADS) {
    const Key mine = keys[k];
    int place = 0;
#pragma unroll 8
    for (int o = 0; o < n; ++o) place += keys[o] > mine;
    if (place < top && mine) out[place] = mine;
  }
}

__device__ __forceinline__ float at_least(float d) { return __builtin_elementwise_maximum(d, kLeast); }  // (a NaN stays one)

// The row's token, asked for before its logits, and that token's logit, asked for once they are there: at the row's end either would be a
// latency to wait for.
__device__ __forceinline__ int token_of(const LogprobArgs& a, int64_t row) { return a.logprob ? a.tokens[row] : -1; }
template <int T>
__device__ __forceinline__ float logit_of(const LogprobArgs& a, int64_t row, int token) {
  if (token < 0 || token >= a.vocab) return -__builtin_inff();
  return (float)reinterpret_cast<const typename Elem<T>::type*>(a.logits)[row * a.stride + token];
}
// unit (x - m), of unit m
__device__ __forceinline__ float below(const LogprobArgs& a, float x, float unit_m) { return __builtin_fmaf(x, a.unit, -unit_m); }
// what a row's outputs are made of, but for the alternatives: by one thread; ln l
__device__ __forceinline__ float finish_row(const LogprobArgs& a, int64_t row, float logit, float m, float l, float w) {
  const float log_l = m == -__builtin_inff() ? __builtin_nanf("") : logf(l);
  if (a.entropy) a.entropy[row] = log_l - w / l * kLn2;
  if (a.logprob) a.logprob[row] = __builtin_fmaf(a.factor, below(a, logit, a.unit * m), -log_l);
  return log_l;
}

__device__ __forceinline__ void store_top(const LogprobArgs& a, int64_t row, int i, Key k, float m, float log_l) {
  a.top_logprob[row * a.top + i] = k ? __builtin_fmaf(a.factor, below(a, value_of(k), a.unit * m), -log_l) : -__builtin_inff();
  a.top_index[row * a.top + i] = k ? index_of(k) : -1;
}

// over the waves, in a fixed order
template <int NW>
__device__ __forceinline__ float max_of(const float* v) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) m = fmaxf(m, v[i]);
  return m;
}
template <int NW>
__device__ __forceinline__ float sum_of(const float* v) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NW; i += 4) s += (v[i] + v[i + 1]) + (v[i + 2] + v[i + 3]);
  return s;
}

// V: vectors of eight values that a thread holds.  grid: row * pieces + piece
template <int T, int V, int THREADS>
__global__ __launch_bounds__(THREADS) void token_logprobs_k(LogprobArgs a) {
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int NW = THREADS / kWave;
  __shared__ float sm_m[NW], sm_l[NW], sm_w[NW], sm_log;
  __shared__ float lane_max[NW][kWave];
  __shared__ int count;
  __shared__ Key listed[kListed], out[kMostTop];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = block_index(), row = b / a.pieces;
  const int piece = (int)(b - row * a.pieces);
  if (row >= a.rows) return;
  const El* x = reinterpret_cast<const El*>(a.logits) + row * a.stride;
  const int vocab = (int)a.vocab, first = piece * (THREADS * 8 * V), token = a.pieces > 1 ? -1 : token_of(a, row);
  float v[V][8], most[V];  // most: of each vector
  if (first + THREADS * 8 * V <= vocab) {  // uniform
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const f32x8 y = E::load8(x + first + (i * THREADS + tid) * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = y[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = first + (i * THREADS + tid) * 8;
      f32x8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = -__builtin_inff();
      if (at + 8 <= vocab) {
        y = E::load8(x + at);
      } else if (at < vocab) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (at + e < vocab) y[e] = (float)x[at + e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = y[e];
    }
  }
  float mine = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    most[i] = v[i][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) most[i] = fmaxf(most[i], v[i][e]);
    mine = fmaxf(mine, most[i]);
  }
  const float logit = logit_of<T>(a, row, token);
  lane_max[wave][lane] = mine;
  const float of_wave = wave_max(mine);
  if (lane == 0) sm_m[wave] = of_wave;
  if (tid == 0) count = 0;
  if (tid < kMostTop) out[tid] = 0;
  __syncthreads();
  const float m = max_of<NW>(sm_m);
  const float m_use = m == -__builtin_inff() ? 0.0f : a.unit * m, c = a.factor * kLog2e;
  float l = 0.0f, w = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = at_least(below(a, v[i][e], m_use) * c), p = __builtin_amdgcn_exp2f(d);
      l += p;
      w = __builtin_fmaf(p, d, w);
    }
  l = wave_sum(l);
  w = wave_sum(w);
  if (lane == 0) {
    sm_l[wave] = l;
    sm_w[wave] = w;
  }
  float low = 0.0f;
  if (a.top > 0) {
    float of_lane = lane_max[0][lane];
#pragma unroll
    for (int i = 1; i < NW; ++i) of_lane = fmaxf(of_lane, lane_max[i][lane]);
    low = value_of(bound_of(order_of(of_lane), a.top));
    if (mine >= low) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!(most[i] >= low)) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (v[i][e] >= low) {
            const int k = atomicAdd(&count, 1);  // (any order: places go by value and index)
            if (k < kListed) listed[k] = key_of(v[i][e], first + (i * THREADS + tid) * 8 + e);
          }
      }
    }
  }
  __syncthreads();
  if (tid == 0) {
    l = sum_of<NW>(sm_l);
    w = sum_of<NW>(sm_w);
    if (a.pieces > 1) a.piece[b] = Piece{m, l, w};
    else sm_log = finish_row(a, row, logit, m, l, w);
  }
  if (a.top == 0) return;
  const int n = count;
  if (n <= kListed) {
    place_keys<THREADS>(listed, n, a.top, out);
  } else {
    // too many share the bound: one at a time, read again, the largest key below the last one taken
    const int end = first + THREADS * 8 * V < vocab ? first + THREADS * 8 * V : vocab;
    Key last = ~(Key)0;
    for (int k = 0; k < a.top; ++k) {
      Key best = 0;
#pragma unroll 1
      for (int here = first + tid; here < end; here += THREADS) {
        const float z = (float)x[here];
        const Key key = z >= low ? key_of(z, here) : 0;
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const Key other = __shfl_xor(best, s, 64);
        best = other > best ? other : best;
      }
      __syncthreads();
      if (lane == 0) listed[wave] = best;
      __syncthreads();
      last = listed[0];
#pragma unroll
      for (int o = 1; o < NW; ++o) last = listed[o] > last ? listed[o] : last;
      if (tid == 0) out[k] = last;
    }
  }
  __syncthreads();
  if (tid < a.top) {
    if (a.pieces > 1) a.best[b * a.top + tid] = out[tid];
    else store_top(a, row, tid, out[tid], m, sm_log);
  }
}

// Joins a row's pieces: a workgroup per row.  The alternatives are among the pieces' own, found as they were found in a piece.
template <int T>
__global__ __launch_bounds__(kPieceThreads) void token_logprobs_join_k(LogprobArgs a) {
  constexpr int NW = kPieceThreads / kWave;
  __shared__ float sm_m[NW], sm_l[NW], sm_w[NW], sm_log;
  __shared__ unsigned lane_max[NW][kWave];
  __shared__ int count;
  __shared__ Key listed[kListed], out[kMostTop];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = block_index();
  if (row >= a.rows) return;
  const int token = token_of(a, row);
  const Piece* piece = a.piece + row * a.pieces;
  const int entries = a.pieces * a.top;
  const Key* best = a.best + row * entries;
  const bool all = entries <= kWave;  // few enough to be listed as they are (32 x 8 of them 10.3 us with, 8 without a bound)
  Key first = tid < entries ? best[tid] : 0;
  Piece p = tid < a.pieces ? piece[tid] : Piece{-__builtin_inff(), 0.0f, 0.0f};
  float m = p.m;
  unsigned mine = (unsigned)(first >> 32);
  for (int i = tid + kPieceThreads; i < a.pieces; i += kPieceThreads) m = fmaxf(m, piece[i].m);
  if (!all)
    for (int i = tid + kPieceThreads; i < entries; i += kPieceThreads) mine = max(mine, (unsigned)(best[i] >> 32));
  const float logit = logit_of<T>(a, row, token);
  m = wave_max(m);
  if (lane == 0) sm_m[wave] = m;
  lane_max[wave][lane] = mine;
  if (tid == 0) count = 0;
  if (tid < kMostTop) out[tid] = 0;
  if (all && tid < kWave) listed[tid] = first;
  __syncthreads();
  m = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
  const float m_use = m == -__builtin_inff() ? 0.0f : a.unit * m, c = a.factor * kLog2e;
  float l = 0.0f, w = 0.0f;
  for (int i = tid; i < a.pieces; i += kPieceThreads) {
    // 2^(d + d') = 2^d 2^d', and (d + d') 2^(d + d') likewise; a piece of nothing has l of 0, or of NaN
    if (i != tid) p = piece[i];
    const float d = at_least(below(a, p.m, m_use) * c), f = __builtin_amdgcn_exp2f(d);
    l = __builtin_fmaf(p.l, f, l);
    w = __builtin_fmaf(f, __builtin_fmaf(p.l, d, p.w), w);
  }
  l = wave_sum(l);
  w = wave_sum(w);
  if (lane == 0) {
    sm_l[wave] = l;
    sm_w[wave] = w;
  }
  int n = entries;
  if (!all) {
    const unsigned low = bound_of(max(max(lane_max[0][lane], lane_max[1][lane]), max(lane_max[2][lane], lane_max[3][lane])), a.top);
    for (int i = tid; i < entries; i += kPieceThreads) {
      const Key k = best[i];
      if ((unsigned)(k >> 32) < low) continue;
      const int at = atomicAdd(&count, 1);
      if (at < kListed) listed[at] = k;
    }
  }
  __syncthreads();
  if (tid == 0) sm_log = finish_row(a, row, logit, m, (sm_l[0] + sm_l[1]) + (sm_l[2] + sm_l[3]), (sm_w[0] + sm_w[1]) + (sm_w[2] + sm_w[3]));
  if (a.top == 0) return;
  if (!all) n = count;
  if (n <= kListed) {
    place_keys<kPieceThreads>(listed, n, a.top, out);
  } else {
    // too many share the bound: one at a time, the largest key below the last one taken
    Key last = ~(Key)0;
    for (int k = 0; k < a.top; ++k) {
      Key most = 0;
      for (int i = tid; i < entries; i += kPieceThreads)
        if (best[i] < last && best[i] > most) most = best[i];
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const Key other = __shfl_xor(most, s, 64);
        most = other > most ? other : most;
      }
      __syncthreads();
      if (lane == 0) listed[wave] = most;
      __syncthreads();
      last = listed[0];
#pragma unroll
      for (int o = 1; o < NW; ++o) last = listed[o] > last ? listed[o] : last;
      if (tid == 0) out[k] = last;
    }
  }
  __syncthreads();
  if (tid < a.top) store_top(a, row, tid, out[tid], m, sm_log);
}

struct LogprobPlan {
  int vectors, threads, pieces;
  size_t ws_bytes;
};
static int plan_logprobs(int64_t rows, int64_t vocab, int type, int top, LogprobPlan& p) {
  if (!known_type(type) || rows < 0 || vocab <= 0 || vocab > kMostVocab || top < 0 || top > kMostTop || mul_overflows(rows, vocab)) return MPQ_ERR_SHAPE;
  auto pieces = [&](int vectors, int threads) { return (vocab + threads * 8 * vectors - 1) / (threads * 8 * vectors); };
  // One piece, the smallest that takes the row, spares the join's launch (us on the device, one piece | several; the host saves 4 more: 1 x
  // 10000 6.1 | 6.6, 100 x 16000 fp32 7.0 | 9.1, 4000 x 10000 fp32 35 | 40).
  p.vectors = 1;
  p.threads = kPieceThreads;
  while (p.vectors < 8 && pieces(p.vectors, p.threads) > 1) p.vectors *= 2;
  if (pieces(8, kPieceThreads) > 1) {
    // Up to 65536 values one workgroup of 16 waves still holds a row, which pays where all rows are on the chip at once: two workgroups to a
    // CU at four vectors, one at eight (one wide piece | several, device: 1 x 32768 bf16 6.0 | 7.2, 256 x 32768 9.1 | 12.7, 512 x 32768
    // 12.3 | 14.9, 1000 x 32768 22.1 | 21.7, 1 x 65536 8.0 | 7.3 but 11.9 | 15.9 from the host, 256 x 60000 fp32 18.7 | 19.7, 512 x 65536
    // bf16 25 | 22).
    const int vectors = pieces(4, kWideThreads) == 1 ? 4 : 8;
    if (pieces(vectors, kWideThreads) == 1 && rows <= 8 * kNumCU / vectors) {
      p.threads = kWideThreads;
      p.vectors = vectors;
    } else {
      // Eight vectors a thread where that makes many rounds of the chip, so that loads overlap with other workgroups' arithmetic, else
      // fewer (2 | 4 | 8 vectors: 2500 x 65536 bf16 92 | 75 | 71, 190 x 100003 fp32 24.2 | 23.1 | 24.0, 1 x 131072 9.1 | 9.6 | 10.4).
      p.vectors = rows * pieces(8, kPieceThreads) >= 8 * kNumCU ? 8 : rows * pieces(4, kPieceThreads) >= 4 * kNumCU ? 4 : 2;
    }
  }
  p.pieces = (int)pieces(p.vectors, p.threads);
  if (mul_overflows(rows, (int64_t)p.pieces * (kMostTop + 4))) return MPQ_ERR_SHAPE;
  p.ws_bytes = p.pieces > 1 ? (size_t)rows * p.pieces * (sizeof(Piece) + (size_t)top * 8) : 0;
  if (rows > 0 && blocks_z(rows * p.pieces, p.threads) > 65535u) return MPQ_ERR_SHAPE;
  return MPQ_OK;
}

template <int T>
static int launch_logprobs(const LogprobArgs& a, const LogprobPlan& p, hipStream_t st) {
  const dim3 grid = wide_grid(a.rows * a.pieces, p.threads);
  if (p.threads == kWideThreads) {
    if (p.vectors == 4) token_logprobs_k<T, 4, kWideThreads><<<grid, kWideThreads, 0, st>>>(a);
    else token_logprobs_k<T, 8, kWideThreads><<<grid, kWideThreads, 0, st>>>(a);
  } else if (p.vectors == 1) {
    token_logprobs_k<T, 1, kPieceThreads><<<grid, kPieceThreads, 0, st>>>(a);
  } else if (p.vectors == 2) {
    token_logprobs_k<T, 2, kPieceThreads><<<grid, kPieceThreads, 0, st>>>(a);
  } else if (p.vectors == 4) {
    token_logprobs_k<T, 4, kPieceThreads><<<grid, kPieceThreads, 0, st>>>(a);
  } else {
    token_logprobs_k<T, 8, kPieceThreads><<<grid, kPieceThreads, 0, st>>>(a);
  }
  const int rc = launch_status();
  if (rc != MPQ_OK || a.pieces == 1) return rc;
  token_logprobs_join_k<T><<<wide_grid(a.rows, kPieceThreads), kPieceThreads, 0, st>>>(a);
  return launch_status();
}

}  // namespace mpq

using namespace mpq;

extern "C" size_t mpq_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int type, int top) {
  LogprobPlan p;
  return plan_logprobs(rows, vocab, type, top, p) == MPQ_OK ? p.ws_bytes : 0;
}

extern "C" int mpq_token_logprobs(const void* logits, int type, int64_t rows, int64_t vocab, int64_t row_stride, float scale,
                                  const int32_t* tokens, float* logprob_out, float* entropy_out, int top, float* top_logprob_out,
                                  int32_t* top_index_out, void* ws, size_t ws_bytes, void* stream) {
  LogprobPlan p;
  const int rc = plan_logprobs(rows, vocab, type, top, p);
  if (rc != MPQ_OK) return rc;
  if (row_stride < vocab || mul_overflows(rows, row_stride) || !(scale > 0.0f) || __builtin_isinf(scale * kLog2e)) return MPQ_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) & (uintptr_t)(type_size(type) - 1)) return MPQ_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(logprob_out) | reinterpret_cast<uintptr_t>(entropy_out)) & 3u)
    return MPQ_ERR_ALIGN;
  if (top > 0 && ((reinterpret_cast<uintptr_t>(top_logprob_out) | reinterpret_cast<uintptr_t>(top_index_out)) & 3u)) return MPQ_ERR_ALIGN;
  if (rows == 0) return MPQ_OK;
  if (!logits || (logprob_out && !tokens) || (top > 0 && (!top_logprob_out || !top_index_out))) return MPQ_ERR_NULL;
  if (!logprob_out && !entropy_out && top == 0) return MPQ_ERR_NULL;
  if (p.ws_bytes > 0 && (!ws || ws_bytes < p.ws_bytes)) return MPQ_ERR_WORKSPACE;
  if (p.ws_bytes > 0 && !aligned16(ws)) return MPQ_ERR_ALIGN;
  int exponent = 0;
  const float half_factor = frexpf(scale, &exponent), unit = scale < 1.0f ? ldexpf(1.0f, exponent - 1) : 1.0f;
  const float factor = scale < 1.0f ? 2.0f * half_factor : scale;
  LogprobArgs a{logits, rows, vocab, row_stride, unit, factor, tokens, logprob_out, entropy_out, top, top_logprob_out, top_index_out, p.pieces,
                nullptr, nullptr};
  if (p.pieces > 1) {
    a.best = reinterpret_cast<Key*>(ws);
    a.piece = reinterpret_cast<Piece*>(a.best + rows * p.pieces * top);
  }
  hipStream_t st = (hipStream_t)stream;
  if (type == MPQ_F32) return launch_logprobs<MPQ_F32>(a, p, st);
  if (type == MPQ_BF16) return launch_logprobs<MPQ_BF16>(a, p, st);
  return launch_logprobs<MPQ_F16>(a, p, st);
}
