// token_logprobs.hip -- log probabilities of given tokens, entropy and the most probable alternatives, from one read of the logits.
//
// With m the row's largest logit, d = scale log2(e) (x - m), l = sum 2^d and w = sum d 2^d:
//   ln p_t = scale (x_t - m) - ln l,   entropy = ln l - ln 2 w / l.
// A workgroup holds a piece of a row in registers, so that the maximum is known before the first exponential and nothing is
// rescaled in the loop.  The largest `top` of a piece: of the 64 maxima of what the four threads of a lane number hold, the
// top-th largest is a bound that at least `top` values reach and few more do; those are listed, and a value's place in the order is
// the number of listed ones before it.  Where too many share the bound (all logits equal, say), they are taken one at a time.
// Rows of several pieces are joined by a wave each.
#include "types.hpp"

namespace mpq {

constexpr int kMostTop = 32, kPieceThreads = 256, kListed = 1024, kJoinListed = 4096;
constexpr int64_t kMostVocab = 1 << 22;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// 2^-200 is 0 in fp32: as the least exponent it leaves minus infinity a product of 0
constexpr float kLeast = -200.0f;

struct Piece {
  float m, l, w;
};
struct LogprobArgs {
  const void* logits;
  int64_t rows, vocab, stride;
  float scale;
  const int32_t* tokens;
  float* logprob;
  float* entropy;
  int top;
  float* top_logprob;
  int32_t* top_index;
  int pieces;
  Piece* piece;       // pieces > 1: [row][piece], then
  float* best;        // [row][piece][top], and
  int32_t* best_at;   // likewise: -1 where there is none
};

// a before b: the larger value, the lower index where they are equal
__device__ __forceinline__ bool before(float a, int ia, float b, int ib) { return a > b || (a == b && ia < ib); }

__device__ __forceinline__ float at_least(float d) { return __builtin_elementwise_maximum(d, kLeast); }  // (a NaN stays one)

// what a row's outputs are made of, but for the alternatives: by one thread; ln l
template <int T>
__device__ __forceinline__ float finish_row(const LogprobArgs& a, int64_t row, float m, float l, float w) {
  const float log_l = m == -__builtin_inff() ? __builtin_nanf("") : logf(l);
  if (a.entropy) a.entropy[row] = log_l - w / l * kLn2;
  if (a.logprob) {
    const int t = a.tokens[row];
    float x = -__builtin_inff();
    if (t >= 0 && t < a.vocab) x = (float)reinterpret_cast<const typename Elem<T>::type*>(a.logits)[row * a.stride + t];
    a.logprob[row] = __builtin_fmaf(a.scale, x - m, -log_l);
  }
  return log_l;
}

// V: vectors of eight values that a thread holds.  grid: row * pieces + piece
template <int T, int V>
__global__ __launch_bounds__(kPieceThreads) void token_logprobs_k(LogprobArgs a) {
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int NW = kPieceThreads / kWave;
  __shared__ float sm_m[NW], sm_l[NW], sm_w[NW], sm_log;
  __shared__ float lane_max[NW][kWave];
  __shared__ float bound;
  __shared__ int count;
  __shared__ float listed[kListed];
  __shared__ int listed_at[kListed];
  __shared__ float out[kMostTop];
  __shared__ int out_at[kMostTop];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = block_index(), row = b / a.pieces;
  const int piece = (int)(b - row * a.pieces);
  if (row >= a.rows) return;
  const El* x = reinterpret_cast<const El*>(a.logits) + row * a.stride;
  const int vocab = (int)a.vocab, first = piece * (kPieceThreads * 8 * V);
  float v[V][8], most[V];  // most: of each vector
  if (first + kPieceThreads * 8 * V <= vocab) {  // uniform
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const f32x8 y = E::load8(x + first + (i * kPieceThreads + tid) * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = y[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = first + (i * kPieceThreads + tid) * 8;
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
  lane_max[wave][lane] = mine;
  const float of_wave = wave_max(mine);
  if (lane == 0) sm_m[wave] = of_wave;
  if (tid == 0) count = 0;
  if (tid < kMostTop) {
    out[tid] = -__builtin_inff();
    out_at[tid] = -1;
  }
  __syncthreads();
  const float m = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
  const float m_use = m == -__builtin_inff() ? 0.0f : m, c = a.scale * kLog2e;
  float l = 0.0f, w = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = at_least((v[i][e] - m_use) * c), p = __builtin_amdgcn_exp2f(d);
      l += p;
      w = __builtin_fmaf(p, d, w);
    }
  l = wave_sum(l);
  w = wave_sum(w);
  if (lane == 0) {
    sm_l[wave] = l;
    sm_w[wave] = w;
  }
  if (a.top > 0 && wave == 0) {
    // the top-th largest of the 64 maxima: its upper 16 bits from the highest down, of a key that orders like the value
    const float of_lane = fmaxf(fmaxf(lane_max[0][lane], lane_max[1][lane]), fmaxf(lane_max[2][lane], lane_max[3][lane]));
    const unsigned u = (unsigned)bits_from_f(of_lane), key = u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
    unsigned at_least = 0;
#pragma unroll 1
    for (unsigned bit = 0x80000000u; bit > 0x8000u; bit >>= 1)
      if (__popcll(__ballot(key >= (at_least | bit))) >= a.top) at_least |= bit;
    // (at least the lowest number, so that minus infinity stays below it; keys below that one are of minus infinity or NaN)
    if (lane == 0) bound = at_least & 0x80000000u ? f_from_bits((int)(at_least ^ 0x80000000u)) : at_least < 0x00800000u ? -__FLT_MAX__ : f_from_bits((int)~at_least);
  }
  __syncthreads();
  l = (sm_l[0] + sm_l[1]) + (sm_l[2] + sm_l[3]);
  w = (sm_w[0] + sm_w[1]) + (sm_w[2] + sm_w[3]);
  if (tid == 0) {
    if (a.pieces > 1) a.piece[b] = Piece{m, l, w};
    else sm_log = finish_row<T>(a, row, m, l, w);
  }
  if (a.top == 0) return;
  const float low = bound;
  if (mine >= low) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (!(most[i] >= low)) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (v[i][e] >= low) {
          const int k = atomicAdd(&count, 1);  // (any order: places go by value and index)
          if (k < kListed) {
            listed[k] = v[i][e];
            listed_at[k] = first + (i * kPieceThreads + tid) * 8 + e;
          }
        }
    }
  }
  __syncthreads();
  const int n = count;
  if (n <= kListed) {
    for (int k = tid; k < n; k += kPieceThreads) {
      const float y = listed[k];
      const int at = listed_at[k];
      int place = 0;
      for (int o = 0; o < n; ++o) place += before(listed[o], listed_at[o], y, at);
      if (place < a.top) {
        out[place] = y;
        out_at[place] = at;
      }
    }
  } else {
    // one at a time, read again: the first in order behind the last one taken
    const int end = first + kPieceThreads * 8 * V < vocab ? first + kPieceThreads * 8 * V : vocab;
    float last = __builtin_inff();
    int last_at = -1;
    for (int k = 0; k < a.top; ++k) {
      float y = -__builtin_inff();
      int at = 0x7FFFFFFF;
#pragma unroll 1
      for (int here = first + tid; here < end; here += kPieceThreads) {
        const float z = (float)x[here];
        if (z >= low && before(last, last_at, z, here) && before(z, here, y, at)) {
          y = z;
          at = here;
        }
      }
      const float top = wave_max(y);
      int low_at = y == top ? at : 0x7FFFFFFF;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) low_at = min(low_at, __shfl_xor(low_at, s, 64));
      __syncthreads();
      if (lane == 0) {
        listed[wave] = top;
        listed_at[wave] = low_at;
      }
      __syncthreads();
      y = listed[0];
      at = listed_at[0];
#pragma unroll
      for (int o = 1; o < NW; ++o)
        if (before(listed[o], listed_at[o], y, at)) {
          y = listed[o];
          at = listed_at[o];
        }
      last = y;
      last_at = at;
      if (tid == 0) {
        out[k] = y;
        out_at[k] = at;
      }
    }
  }
  __syncthreads();
  if (tid < a.top) {
    if (a.pieces > 1) {
      a.best[b * a.top + tid] = out[tid];
      a.best_at[b * a.top + tid] = out_at[tid];
    } else {
      a.top_logprob[row * a.top + tid] = out_at[tid] < 0 ? -__builtin_inff() : __builtin_fmaf(a.scale, out[tid] - m, -sm_log);
      a.top_index[row * a.top + tid] = out_at[tid];
    }
  }
}

// Joins a row's pieces: a wave per row.  The pieces' lists are in order, so that the next alternative is the first of their heads.
template <int T>
__global__ __launch_bounds__(kWave) void token_logprobs_join_k(LogprobArgs a) {
  extern __shared__ int lds[];  // of each piece, how many of its list were taken; the lists where they fit
  const int lane = threadIdx.x;
  const int64_t row = block_index();
  if (row >= a.rows) return;
  const Piece* piece = a.piece + row * a.pieces;
  float m = -__builtin_inff();
  for (int i = lane; i < a.pieces; i += kWave) m = fmaxf(m, piece[i].m);
  m = wave_max(m);
  const float m_use = m == -__builtin_inff() ? 0.0f : m, c = a.scale * kLog2e;
  float l = 0.0f, w = 0.0f;
  for (int i = lane; i < a.pieces; i += kWave) {
    // 2^(d + d') = 2^d 2^d', and (d + d') 2^(d + d') likewise; a piece of nothing has l of 0, or of NaN
    const Piece p = piece[i];
    const float d = at_least((p.m - m_use) * c), f = __builtin_amdgcn_exp2f(d);
    l = __builtin_fmaf(p.l, f, l);
    w = __builtin_fmaf(f, __builtin_fmaf(p.l, d, p.w), w);
  }
  l = wave_sum(l);
  w = wave_sum(w);
  float log_l = 0.0f;
  if (lane == 0) log_l = finish_row<T>(a, row, m, l, w);
  if (a.top == 0) return;
  log_l = __shfl(log_l, 0, 64);
  const int entries = a.pieces * a.top;
  const float* best = a.best + row * entries;
  const int32_t* best_at = a.best_at + row * entries;
  int* head = lds;
  for (int i = lane; i < a.pieces; i += kWave) head[i] = 0;
  if (entries <= kJoinListed) {
    int *to_at = lds + a.pieces, *to = to_at + entries;
    for (int i = lane; i < entries; i += kWave) {
      to[i] = bits_from_f(best[i]);
      to_at[i] = best_at[i];
    }
    best = reinterpret_cast<float*>(to);
    best_at = to_at;
  }
  __syncthreads();
  // the first of the heads of the lane's pieces, looked for again only where it was taken
  float y;
  int at, of;
  auto look = [&]() {
    y = -__builtin_inff();
    at = 0x7FFFFFFF;
    for (int i = lane; i < a.pieces; i += kWave) {
      const int h = head[i];
      if (h >= a.top) continue;
      const float z = best[i * a.top + h];
      const int z_at = best_at[i * a.top + h];
      if (z_at >= 0 && before(z, z_at, y, at)) {
        y = z;
        at = z_at;
        of = i;
      }
    }
  };
  look();
  for (int k = 0; k < a.top; ++k) {
    const float most = wave_max(y);
    int low = y == most ? at : 0x7FFFFFFF;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) low = min(low, __shfl_xor(low, s, 64));
    const bool any = low != 0x7FFFFFFF;
    if (lane == 0) {
      a.top_logprob[row * a.top + k] = any ? __builtin_fmaf(a.scale, most - m, -log_l) : -__builtin_inff();
      a.top_index[row * a.top + k] = any ? low : -1;
    }
    if (any && at == low) {  // (an index is in one piece)
      head[of] += 1;
      look();
    }
  }
}

struct LogprobPlan {
  int vectors, pieces;
  size_t ws_bytes;
};
static int plan_logprobs(int64_t rows, int64_t vocab, int type, int top, LogprobPlan& p) {
  if (!known_type(type) || rows < 0 || vocab <= 0 || vocab > kMostVocab || top < 0 || top > kMostTop) return MPQ_ERR_SHAPE;
  auto pieces = [&](int vectors) { return (vocab + kPieceThreads * 8 * vectors - 1) / (kPieceThreads * 8 * vectors); };
  p.vectors = 8;
  while (p.vectors > 1 && (rows * pieces(p.vectors) < 2 * kNumCU || pieces(p.vectors / 2) == 1)) p.vectors /= 2;
  p.pieces = (int)pieces(p.vectors);
  if (mul_overflows(rows, (int64_t)p.pieces * (kMostTop + 4))) return MPQ_ERR_SHAPE;
  p.ws_bytes = p.pieces > 1 ? (size_t)rows * p.pieces * (sizeof(Piece) + (size_t)top * 8) : 0;
  if (rows > 0 && blocks_z(rows * p.pieces, kPieceThreads) > 65535u) return MPQ_ERR_SHAPE;
  return MPQ_OK;
}

template <int T>
static int launch_logprobs(const LogprobArgs& a, const LogprobPlan& p, hipStream_t st) {
  const dim3 grid = wide_grid(a.rows * a.pieces, kPieceThreads);
  if (p.vectors == 1) token_logprobs_k<T, 1><<<grid, kPieceThreads, 0, st>>>(a);
  else if (p.vectors == 2) token_logprobs_k<T, 2><<<grid, kPieceThreads, 0, st>>>(a);
  else if (p.vectors == 4) token_logprobs_k<T, 4><<<grid, kPieceThreads, 0, st>>>(a);
  else token_logprobs_k<T, 8><<<grid, kPieceThreads, 0, st>>>(a);
  const int rc = launch_status();
  if (rc != MPQ_OK || a.pieces == 1) return rc;
  const int lists = a.pieces * a.top <= kJoinListed ? a.pieces * a.top : 0;
  token_logprobs_join_k<T><<<wide_grid(a.rows, kWave), kWave, (a.pieces + 2 * lists) * sizeof(int), st>>>(a);
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
  if (row_stride < vocab || mul_overflows(rows, row_stride) || !(scale > 0.0f) || __builtin_isinf(scale)) return MPQ_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(logits) & (uintptr_t)(type_size(type) - 1)) return MPQ_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(logprob_out) | reinterpret_cast<uintptr_t>(entropy_out)) & 3u)
    return MPQ_ERR_ALIGN;
  if (top > 0 && ((reinterpret_cast<uintptr_t>(top_logprob_out) | reinterpret_cast<uintptr_t>(top_index_out)) & 3u)) return MPQ_ERR_ALIGN;
  if (rows == 0) return MPQ_OK;
  if (!logits || (logprob_out && !tokens) || (top > 0 && (!top_logprob_out || !top_index_out))) return MPQ_ERR_NULL;
  if (!logprob_out && !entropy_out && top == 0) return MPQ_ERR_NULL;
  if (p.ws_bytes > 0 && (!ws || ws_bytes < p.ws_bytes)) return MPQ_ERR_WORKSPACE;
  if (p.ws_bytes > 0 && !aligned16(ws)) return MPQ_ERR_ALIGN;
  LogprobArgs a{logits, rows, vocab, row_stride, scale, tokens, logprob_out, entropy_out, top, top_logprob_out, top_index_out, p.pieces,
                nullptr, nullptr, nullptr};
  if (p.pieces > 1) {
    a.piece = reinterpret_cast<Piece*>(ws);
    a.best = reinterpret_cast<float*>(a.piece + rows * p.pieces);
    a.best_at = reinterpret_cast<int32_t*>(a.best + rows * p.pieces * top);
  }
  hipStream_t st = (hipStream_t)stream;
  if (type == MPQ_F32) return launch_logprobs<MPQ_F32>(a, p, st);
  if (type == MPQ_BF16) return launch_logprobs<MPQ_BF16>(a, p, st);
  return launch_logprobs<MPQ_F16>(a, p, st);
}
