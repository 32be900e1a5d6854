// linear_groups.hip -- a linear layer of few rows whose 4-bit weights have a step per group of 32, 64 or 128 input channels.
//
// y[m][n] = act(sum_g s[n][g] sum_{k in g} c[n][k] x[m][k]).  The weights are read once and meet at most 64 rows at a time, so that their bytes
// bound it while there are few rows (1 x 4096 x 12288, fp16 steps: 26 MB in 8.4 us, of which a launch takes 2.6; a kernel that only reads
// so many in the same way takes 5.3).  With many rows it is latency: 61 x 4096 x 11008, groups of 32, takes 19.7 us, of whose cycles vector instructions
// fill 34 % and matrix steps 9 %.  One to two waves to a SIMD wait for a chain -- a matrix step's rows from LDS, the product, the product times the
// steps -- that a scheduling barrier keeps apart from the next one's, and 230 workgroups read 115 MB of x out of the L2 (the loads alone: 17 us).
// A lane loads 16 bytes, 32 codes, of a weight row; the waves of a workgroup share k out among them and their sums meet in LDS, in a
// fixed order.
//
// The product runs on v_mfma_f32_16x16x32 in the rows' own 16-bit type (rows x times codes): bf16 and fp16 hold x and codes exactly.
// fp32 rows go in as three bf16 terms, 24 bits.  Operands are the codes themselves, so that a sum holds nothing but the products.  (Cheaper to make is
// code + 24, the code's bits in the mantissa of 16, and -24 times the group's sum of x added in again: rows of one sign then lose four bits of
// fp32 -- K = 4096, rows behind a ReLU, groups of 128: 5e-6 of the outputs' norm -- for times within 4 % of these, but for one row of bf16 with fp32
// steps, 1 x 4096 x 12288 in groups of 64, 8.5 us against 9.3.)  fp16: that form, less 24 in one packed instruction for two codes.  bf16, which
// has no such instruction: v_cvt_off_f32_i4 makes code / 16 of four bits, whose upper half is the operand; the 16 is
// multiplied in at the end, so that outputs within 2^4 of the least normal number may lose as many bits.
//
// A group's sum has to hold that group alone, and a matrix step adds up the k of four quarters of the wave.  A lane's 16 bytes are
// 32 neighbouring codes: the quarters exchange their dwords, four swaps for four dwords, after which dword c has 32 neighbouring k.
#include "qgemm_dma.hpp"

#include <type_traits>

namespace mpq {

struct GroupsArgs {
  const void* x;
  int64_t x_stride;
  const uint8_t* w;
  const void* scale;
  int64_t M, N;
  int K, scale_type, act, y_type;
  void* y;
};

constexpr int kGroupWaves = 8, kGroupThreads = kGroupWaves * 64;

// UNIT: what operands of codes are counted in
template <int T>
struct Operand {  // bf16, also for the terms of fp32
  static constexpr int TERMS = T == MPQ_F32 ? 3 : 1;
  static constexpr float UNIT = 16.0f;
  static __device__ __forceinline__ f32x4 mfma(v4i a, v4i b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  // eight codes as an operand: its dword i holds codes i and i + 4
  static __device__ __forceinline__ v4i codes(unsigned w) {
    const unsigned odd = w >> 4;
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned of = i & 1 ? odd : w;
      const float low = __builtin_amdgcn_cvt_off_f32_i4(of >> 8 * (i >> 1)), high = __builtin_amdgcn_cvt_off_f32_i4(of >> (8 * (i >> 1) + 16));
      r[i] = (int)__builtin_amdgcn_perm((unsigned)bits_from_f(high), (unsigned)bits_from_f(low), 0x07060302u);
    }
    return r;
  }
};
template <>
struct Operand<MPQ_F16> {
  static constexpr int TERMS = 1;
  static constexpr float UNIT = 1.0f;
  static __device__ __forceinline__ f32x4 mfma(v4i a, v4i b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  // 16, and the code's sign bit turned in the mantissa behind it: code + 24, less that
  static __device__ __forceinline__ v4i codes(unsigned w) {
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int left = 6 - 4 * i;
      const unsigned v = left >= 0 ? w << (left & 31) : w >> (-left & 31);
      const f16x2 with = __builtin_bit_cast(f16x2, (v & 0x03C003C0u) ^ (0x4C004C00u ^ 0x02000200u));
      r[i] = __builtin_bit_cast(int, with - f16x2{(_Float16)24, (_Float16)24});
    }
    return r;
  }
};
// eight 16-bit values in their order -> the order of Operand::codes
__device__ __forceinline__ v4i pair_up(v4i v) {
  return v4i{(int)__builtin_amdgcn_perm((unsigned)v.z, (unsigned)v.x, 0x05040100u), (int)__builtin_amdgcn_perm((unsigned)v.z, (unsigned)v.x, 0x07060302u),
             (int)__builtin_amdgcn_perm((unsigned)v.w, (unsigned)v.y, 0x05040100u), (int)__builtin_amdgcn_perm((unsigned)v.w, (unsigned)v.y, 0x07060302u)};
}

// eight values of x as they are loaded, and as operands
template <int T>
struct Values {
  typedef v4i type;
  static __device__ __forceinline__ v4i load(const typename Elem<T>::type* p) { return *reinterpret_cast<const v4i_byte*>(p); }
  static __device__ __forceinline__ void split(v4i v, v4i (&term)[1]) { term[0] = pair_up(v); }
};
template <>
struct Values<MPQ_F32> {
  typedef f32x8 type;
  static __device__ __forceinline__ f32x8 load(const float* p) { return Elem<MPQ_F32>::load8(p); }
  static __device__ __forceinline__ void split(f32x8 v, v4i (&term)[3]) {
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      const bf16x8 top = __builtin_convertvector(v, bf16x8);
      term[t] = pair_up(__builtin_bit_cast(v4i, top));
      v -= __builtin_convertvector(top, f32x8);
    }
  }
};

// Dword d of quarter c becomes dword c of quarter d.
__device__ __forceinline__ v4i exchange(v4i v) {
  const auto a = __builtin_amdgcn_permlane32_swap((unsigned)v.x, (unsigned)v.z, false, false);
  const auto b = __builtin_amdgcn_permlane32_swap((unsigned)v.y, (unsigned)v.w, false, false);
  const auto c = __builtin_amdgcn_permlane16_swap((unsigned)a[0], (unsigned)b[0], false, false);
  const auto d = __builtin_amdgcn_permlane16_swap((unsigned)a[1], (unsigned)b[1], false, false);
  return v4i{(int)c[0], (int)c[1], (int)d[0], (int)d[1]};
}

// COUNT neighbouring steps of 4 or 2 bytes, at any address that one may have
template <bool WIDE, int COUNT>
struct Steps {
  typedef typename std::conditional<WIDE, float, unsigned short>::type El;
  typedef El Raw __attribute__((ext_vector_type(COUNT)));
  typedef El RawAny __attribute__((ext_vector_type(COUNT), aligned(sizeof(El))));
  Raw v;
  __device__ __forceinline__ void load(const void* p, int64_t at) { v = *reinterpret_cast<const RawAny*>(reinterpret_cast<const El*>(p) + at); }
  // bf16: all bits set where the 2 bytes are one, else none (a choice in bits: at a branch the compiler would keep everything in registers)
  __device__ __forceinline__ float get(int i, unsigned bf16) const {
    if constexpr (WIDE) return v[i];
    else return f_from_bits((int)(((unsigned)v[i] << 16 & bf16) | ((unsigned)bits_from_f((float)__builtin_bit_cast(_Float16, (unsigned short)v[i])) & ~bf16)));
  }
};

// The waves' sums of MT row tiles, in a fixed order, times unit to y: lane (channel, rows 4 q .. 4 q + 3).  m0, rows: of the first tile.
template <int MT, int NT>
__device__ __forceinline__ void store_tiles(const GroupsArgs& p, f32x4* red, const f32x4 (*total)[NT], int64_t m0, int rows, int64_t n0, float unit) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) red[((wave * MT + i) * NT + j) * 64 + lane] = total[i][j];
  __syncthreads();
  for (int t = threadIdx.x; t < MT * NT * 64; t += kGroupThreads) {
    const int tile = t >> 6, i = tile / NT, j = tile % NT, l = t & 63;
    f32x4 sum = red[t];
#pragma unroll
    for (int v = 1; v < kGroupWaves; ++v) sum += red[v * (MT * NT * 64) + t];
    const int64_t n = n0 + j * 16 + (l & 15);
    if (n >= p.N) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int m = i * 16 + 4 * (l >> 4) + e;
      if (m >= rows) continue;
      const float y = apply_act(sum[e] * unit, p.act);
      const int64_t to = (m0 + m) * p.N + n;
      if (p.y_type == MPQ_F32) reinterpret_cast<float*>(p.y)[to] = y;
      else reinterpret_cast<unsigned short*>(p.y)[to] = to_half(y, p.y_type == MPQ_BF16);
    }
  }
}

// What the two kernels share: the sums of 64 k, `half` of a step of 128, times their groups' steps to the totals.  `term` holds x of 32 k as
// operands, of MT row tiles.  Groups of 128 are summed over both halves.
template <int T, int MT, int NT, int G>
struct HalfSums {
  using O = Operand<T>;
  static constexpr int PER = G / 32;
  f32x4 part[PER > 1 ? NT : 1][MT];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < (PER > 1 ? NT : 1); ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) part[j][i] = f32x4{0, 0, 0, 0};
  }
  // to part j, or its first: 32 k
  __device__ __forceinline__ void product(const v4i (&term)[MT][O::TERMS], unsigned w, int j, bool first) {
    const v4i codes = O::codes(w);
#pragma unroll
    for (int t = 0; t < O::TERMS; ++t)
#pragma unroll
      for (int i = 0; i < MT; ++i) part[j][i] = O::mfma(term[i][t], codes, first && t == 0 ? f32x4{0, 0, 0, 0} : part[j][i]);
  }
  __device__ __forceinline__ void scale(f32x4 (&total)[MT][NT], int j, float step) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) total[i][j][e] = __builtin_fmaf(part[PER > 1 ? j : 0][i][e], step, total[i][j][e]);
  }
  // term_of(c, term), dword c of a half's codes w[j][c], step_of(j, c): of tile j, of the group that ends with c; there: matrix steps of
  // the half, 1 or 2; last: whether a group of 128 ends
  template <typename TermOf, typename WOf, typename StepOf>
  __device__ __forceinline__ void add(f32x4 (&total)[MT][NT], int there, bool last, TermOf&& term_of, WOf&& w_of, StepOf&& step_of) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (c >= there) break;  // uniform
      __builtin_amdgcn_sched_barrier(0);  // (matrix steps stay apart: drawn into one another they would not fit the registers)
      v4i term[MT][O::TERMS];
      term_of(c, term);
      unsigned w[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = w_of(j, c);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        product(term, w[j], PER > 1 ? j : 0, PER == 1 || (PER == 2 && c == 0));
        if (PER == 1) scale(total, j, step_of(j, c));
      }
      if (PER == 2 && c == 1) {
#pragma unroll
        for (int j = 0; j < NT; ++j) scale(total, j, step_of(j, 0));
      }
    }
    if (PER == 4 && last) {
#pragma unroll
      for (int j = 0; j < NT; ++j) scale(total, j, step_of(j, 0));
      clear();
    }
  }
};

// T: type of x, WIDE: steps of 4 bytes, G: group.  A workgroup takes NT x 16 output channels and MT x 16 rows, its waves steps of 128 k.
// A wave's rows of x come 64 k at a time, whole cache lines, through registers into LDS of its own, from where a lane reads its row's operands:
// read straight as operands, 16 rows of 64 bytes a time, a line came twice (64 x 4096 x 11008, groups of 128: 55 us with a channel tile to a
// workgroup, 30 so, 18 with three).
// grid: x channels, y blocks of rows
template <int T, bool WIDE, int G, int MT, int NT>
__global__ __launch_bounds__(kGroupThreads, 2) void linear_groups_k(GroupsArgs p) {
  typedef typename Elem<T>::type El;
  constexpr int NW = kGroupWaves, TERMS = Operand<T>::TERMS, STEP = 128, OF_STEP = STEP / G;  // groups of a step
  constexpr int CH = 64 * (int)sizeof(El) / 16;            // chunks of 16 bytes of a row and 64 k
  constexpr int LOADS = MT * 16 * CH / 64;                 // a lane's
  constexpr int PASS = MT < 2 ? 1 : 2;                     // row tiles whose sums meet in LDS together
  constexpr int STAGE = NW * MT * 16 * CH, RED = NW * PASS * NT * 64;
  __shared__ v4i lds[STAGE > RED ? STAGE : RED];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, q = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT), m0 = (int64_t)blockIdx.y * (16 * MT);
  const int K = p.K, groups = K / G;
  const int rows = (int)(p.M - m0 < 16 * MT ? p.M - m0 : 16 * MT);
  const unsigned bf16_steps = p.scale_type == MPQ_BF16 ? ~0u : 0u;
  // channels and rows past the edge re-read the last one; never stored
  const uint8_t* w_row[NT];
  int64_t s_row[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t n = n0 + j * 16 + r < p.N ? n0 + j * 16 + r : p.N - 1;
    w_row[j] = p.w + n * (K >> 1);
    s_row[j] = n * groups;
  }
  // the lane's loads of x: row and chunk
  const El* x_row[LOADS];
  v4i* own = lds + wave * (MT * 16 * CH);
  int put[LOADS];
  constexpr int EL = 16 / (int)sizeof(El);
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = (i * 64 + lane) / CH, chunk = lane % CH;
    x_row[i] = reinterpret_cast<const El*>(p.x) + (m0 + (row < rows ? row : rows - 1)) * p.x_stride + chunk * EL;
    put[i] = row * CH + (chunk ^ (row >> 1 & 7));  // (so that 16 rows' reads of one chunk fall into different banks)
  }
  auto read = [&](int i, int chunk) {
    const int row = i * 16 + r;
    return own[row * CH + (chunk ^ (row >> 1 & 7))];
  };

  // Whole steps are dealt out to the waves in turn, so that neighbours read a line's two halves of codes, and the lines of their steps, at about the
  // same time (a piece of k to each: 16 x 4096 x 11008, groups of 32, takes 7 % more, 64 rows alike).  What comes next is requested while this is multiplied, without a branch: behind one the compiler
  // does not know what is in flight, and waits for everything.  Loads arrive in the order of their requests, so that whatever was requested
  // before something that is waited for has been waited for as well.
  const int whole = K / STEP;
  f32x4 total[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) total[i][j] = f32x4{0, 0, 0, 0};
  HalfSums<T, MT, NT, G> sums;
  sums.clear();
  auto request_x = [&](v4i (&to)[LOADS], int k) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) to[i] = *reinterpret_cast<const v4i_byte*>(x_row[i] + k);
  };
  struct Weights {
    v4i w[NT];
    Steps<WIDE, OF_STEP> sc[NT];
  };
  auto request_w = [&](Weights& to, int s) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      to.w[j] = *reinterpret_cast<const v4i_byte*>(w_row[j] + ((s * STEP + 32 * q) >> 1));
      to.sc[j].load(p.scale, s_row[j] + s * OF_STEP);
    }
  };
  auto arrange = [&](Weights& of) {
#pragma unroll
    for (int j = 0; j < NT; ++j) of.w[j] = exchange(of.w[j]);
  };
  auto stage = [&](const v4i (&x)[LOADS]) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // what the lanes read of the last one has been read
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) own[put[i]] = x[i];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  auto term_of = [&](int c, v4i (&term)[MT][TERMS]) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int chunk = c * (CH / 2) + q * (CH / 8);
      if constexpr (T == MPQ_F32) {
        const f32x4 a = __builtin_bit_cast(f32x4, read(i, chunk)), b = __builtin_bit_cast(f32x4, read(i, chunk + 1));
        Values<T>::split(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), term[i]);
      } else {
        Values<T>::split(read(i, chunk), term[i]);
      }
    }
  };
  auto multiply = [&](const Weights& of, int half, int there, bool last) {
    sums.add(total, there, last, term_of, [&](int j, int c) { return (unsigned)of.w[j][2 * half + c]; },
             [&](int j, int c) { return of.sc[j].get(G == 32 ? 2 * half + c : G == 64 ? half : 0, bf16_steps); });
  };
  // rows a half step ahead, weights a step, behind the rows that are waited for first (all of one or two steps ahead, where rows are few enough for the
  // registers, was no faster: 16 x 4096 x 11008, groups of 32, takes 17 % more)
  if (wave < whole) {
    v4i x[LOADS];
    Weights now, next;
    request_x(x, wave * STEP);
    request_w(now, wave);
#pragma unroll 1
    for (int s = wave; s < whole; s += NW) {
      const int then = s + NW < whole ? s + NW : s;
      arrange(now);
      stage(x);
      request_x(x, s * STEP + 64);
      request_w(next, then);
      multiply(now, 0, 2, false);
      stage(x);
      request_x(x, then * STEP);
      multiply(now, 1, 2, true);
      now = next;
    }
  }
  if (G < 128 && whole * STEP < K && wave == NW - 1) {  // the rest of the row: one to three matrix steps
    // a lane's 32 codes, and its chunk of x, lie in the row or behind it, as a whole; those behind are not multiplied
    const int k = whole * STEP, there = (K - k) / 32, at = k + 32 * q;
    v4i x[LOADS];
    Weights rest;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      rest.w[j] = *reinterpret_cast<const v4i_byte*>(w_row[j] + ((at < K ? at : K - 32) >> 1));
#pragma unroll
      for (int g = 0; g < OF_STEP; ++g) {
        Steps<WIDE, 1> one;
        one.load(p.scale, s_row[j] + (whole * OF_STEP + g < groups ? whole * OF_STEP + g : groups - 1));
        rest.sc[j].v[g] = one.v[0];
      }
    }
    arrange(rest);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (2 * half >= there) break;  // uniform
      const int first = lane % CH * EL, here = k + 64 * half;
      request_x(x, here + first < K ? here : K - EL - first);
      stage(x);
      multiply(rest, half, there - 2 * half, false);
    }
  }
  __syncthreads();  // the waves' sums go where x was
#pragma unroll
  for (int i = 0; i < MT; i += PASS) {
    if (i) __syncthreads();
    store_tiles<PASS, NT>(p, reinterpret_cast<f32x4*>(lds), total + i, m0 + 16 * i, rows - 16 * i, n0, Operand<T>::UNIT);
  }
}

// Few rows: x as a whole in LDS, as operands, and the steps of the workgroup's channels, which lie together in memory, beside it.  Read
// straight as operands, x would come with 16 times the loads that it is long, and steps in pieces of 2 bytes a line: a CU has a line from the L2 in
// four clocks at best, and its lines bound it (1 x 4096 x 12288, fp16 steps, groups of 128: 12.2 us so).
// Four units of 128 k of a wave are in flight, and once they have arrived the next four.  LDS: [row][k / 8][term], rows 64 bytes apart
// modulo 256; [channel][group].
constexpr int kUnits = 4, kFewRows = 8;
__host__ __device__ inline int x_row_chunks(int K, int terms) {
  const int n = K / 8 * terms;
  return n + (4 - n % 16 + 16) % 16;
}
// steps from a channel to the next there: 16 bytes further where channels are whole pieces of 16, so that 16 of them fall into different banks
__host__ __device__ inline int step_row_length(int groups, int step_size) { return groups * step_size % 16 ? groups : groups + 16 / step_size; }
// bytes of LDS of a call: x, whose place the waves' sums take, and steps; the latter alone
inline int few_steps_bytes(int64_t K, int group, int step_size) { return (16 * step_row_length((int)(K / group), step_size) * step_size + 15) / 16 * 16; }
inline int64_t few_bytes(int64_t M, int64_t K, int terms, int group, int step_size) {
  if (M > kFewRows || K > (1 << 16)) return 1 << 30;
  const int64_t x = M * x_row_chunks((int)K, terms) * 16, red = kGroupWaves * 1024;
  return (x > red ? x : red) + few_steps_bytes(K, group, step_size);
}
template <int T, bool WIDE, int G>
__global__ __launch_bounds__(kGroupThreads) void linear_groups_few_k(GroupsArgs p, int x_bytes) {
  constexpr int NT = 1;
  typedef typename Elem<T>::type El;
  typedef typename Steps<WIDE, 1>::El StepEl;
  constexpr int NW = kGroupWaves, TERMS = Operand<T>::TERMS, UNIT = 128, OF_UNIT = UNIT / G;
  extern __shared__ v4i few_lds[];
  StepEl* steps = reinterpret_cast<StepEl*>(reinterpret_cast<char*>(few_lds) + x_bytes);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const int r = lane & 15, q = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
  const int K = p.K, groups = K / G, rows = (int)p.M, row_chunks = x_row_chunks(K, TERMS), per_row = K / 8, chunks = rows * per_row;
  const unsigned bf16_steps = p.scale_type == MPQ_BF16 ? ~0u : 0u;
  // this thread's first pieces of x and of the steps are requested before the weights, and stored behind their request
  auto load_x = [&](int i, int& to) {
    const int row = rows == 1 ? 0 : i / per_row, chunk = i - row * per_row;
    to = row * row_chunks + chunk * TERMS;
    return Values<T>::load(reinterpret_cast<const El*>(p.x) + row * p.x_stride + chunk * 8);
  };
  auto store_x = [&](typename Values<T>::type v, int to) {
    v4i term[TERMS];
    Values<T>::split(v, term);
#pragma unroll
    for (int t = 0; t < TERMS; ++t) few_lds[to + t] = term[t];
  };
  const int channels = (int)(p.N - n0 < 16 * NT ? p.N - n0 : 16 * NT);
  const StepEl* step_from = reinterpret_cast<const StepEl*>(p.scale) + n0 * groups;
  constexpr int SE = 16 / (int)sizeof(StepEl);
  const int step_count = channels * groups, step_chunks = step_count / SE;
  int x_to = 0;
  typename Values<T>::type x_first = typename Values<T>::type{};
  v4i s_first = {0, 0, 0, 0};
  if (tid < chunks) x_first = load_x(tid, x_to);
  if (tid < step_chunks) s_first = *reinterpret_cast<const v4i_byte*>(step_from + tid * SE);
  // channels past the edge re-read the last one; never stored
  const uint8_t* w_row[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) w_row[j] = p.w + (n0 + (j * 16 + r < channels ? j * 16 + r : channels - 1)) * (K >> 1) + 16 * q;
  // units are dealt out to the waves as linear_groups_k deals its steps: a row's sums are the same, bit for bit, in both kernels
  const int whole = K / UNIT;
  v4i w[kUnits][NT], w_next[kUnits][NT];
  auto request = [&](v4i (&to)[kUnits][NT], int s) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = s + u * NW < whole ? s + u * NW : whole - 1;
#pragma unroll
      for (int j = 0; j < NT; ++j) to[u][j] = *reinterpret_cast<const v4i_byte*>(w_row[j] + at * (UNIT / 2));
    }
  };
  if (wave < whole) request(w, wave);
  if (tid < chunks) store_x(x_first, x_to);
  const int row_length = step_row_length(groups, sizeof(StepEl));
  auto store_steps = [&](v4i v, int i) {
    if (row_length != groups) i += i / (groups / SE);
    reinterpret_cast<v4i*>(steps)[i] = v;
  };
  if (tid < step_chunks) store_steps(s_first, tid);
#pragma unroll 1
  for (int i = tid + kGroupThreads; i < chunks; i += kGroupThreads) {
    int to;
    const auto v = load_x(i, to);
    store_x(v, to);
  }
#pragma unroll 1
  for (int i = tid + kGroupThreads; i < step_chunks; i += kGroupThreads) store_steps(*reinterpret_cast<const v4i_byte*>(step_from + i * SE), i);
  if (tid < step_count - step_chunks * SE) steps[step_chunks * SE + tid] = step_from[step_chunks * SE + tid];
  __syncthreads();
  const v4i* x_row = few_lds + (r < rows ? r : 0) * row_chunks + q * TERMS;  // (rows past the edge: never stored)
  f32x4 total[1][NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) total[0][j] = f32x4{0, 0, 0, 0};
  HalfSums<T, 1, NT, G> sums;
  sums.clear();
  int step_row[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) step_row[j] = (j * 16 + r < channels ? j * 16 + r : channels - 1) * row_length;
  auto unit = [&](v4i (&codes)[NT], int s, int there) {
#pragma unroll
    for (int j = 0; j < NT; ++j) codes[j] = exchange(codes[j]);
    const v4i* x = x_row + s * (UNIT / 8) * TERMS;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (2 * half >= there) break;  // uniform
      sums.add(total, there - 2 * half, half == 1, [&](int c, v4i (&term)[1][TERMS]) {
#pragma unroll
        for (int t = 0; t < TERMS; ++t) term[0][t] = x[(8 * half + 4 * c) * TERMS + t];
      }, [&](int j, int c) { return (unsigned)codes[j][2 * half + c]; }, [&](int j, int c) {
        Steps<WIDE, 1> one;
        one.v[0] = steps[step_row[j] + s * OF_UNIT + (G == 32 ? 2 * half + c : G == 64 ? half : 0)];
        return one.get(0, bf16_steps);
      });
    }
  };
  // (the last units apart, so that the loop needs no branch around its requests)
  int s = wave;
#pragma unroll 1
  for (; s + kUnits * NW < whole; s += kUnits * NW) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int j = 0; j < NT; ++j) asm volatile("" : "+v"(w[u][j]));  // here they have arrived: a wait further down would be one for the next as well
    request(w_next, s + kUnits * NW);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) unit(w[u], s + u * NW, 4);
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int j = 0; j < NT; ++j) w[u][j] = w_next[u][j];
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (s + u * NW >= whole) break;  // uniform
    unit(w[u], s + u * NW, 4);
  }
  if (G < 128 && whole * UNIT < K && wave == NW - 1) {  // the rest of the row: one to three matrix steps
    // a lane's 32 codes lie in the row or behind it, as a whole; those behind are not multiplied
    const int at = whole * UNIT + 32 * q;
#pragma unroll
    for (int j = 0; j < NT; ++j) w[0][j] = *reinterpret_cast<const v4i_byte*>(w_row[j] - 16 * q + ((at < K ? at : K - 32) >> 1));
    unit(w[0], whole, (K - whole * UNIT) / 32);
  }
  __syncthreads();  // the waves' sums go where x was
  store_tiles<1, NT>(p, reinterpret_cast<f32x4*>(few_lds), total, 0, rows, n0, Operand<T>::UNIT);
}

// Channel tiles per workgroup: what makes the bytes that a CU loads smallest, its workgroups' weights and rows.
static int channel_tiles(int mt, const GroupsArgs& p, int el) {
  int best = 1;
  double least = 0;
  for (int nt = 1; nt <= 3; ++nt) {
    const int64_t workgroups = (p.N + 16 * nt - 1) / (16 * nt), rounds = (workgroups * ((p.M + 16 * mt - 1) / (16 * mt)) + kNumCU - 1) / kNumCU;
    const double bytes = (double)rounds * (nt * 16 * 0.5 + (p.M < 16 * mt ? p.M : 16 * mt) * el);
    if (nt == 1 || bytes < least) { least = bytes; best = nt; }
  }
  return best;
}

template <int T, bool WIDE, int G, int MT>
static int go(const GroupsArgs& p, hipStream_t st) {
  const int nt = channel_tiles(MT, p, T == MPQ_F32 ? 4 : 2);
  const dim3 grid((unsigned)((p.N + 16 * nt - 1) / (16 * nt)), (unsigned)((p.M + 16 * MT - 1) / (16 * MT)));
  if (nt == 1) linear_groups_k<T, WIDE, G, MT, 1><<<grid, kGroupThreads, 0, st>>>(p);
  else if (nt == 2) linear_groups_k<T, WIDE, G, MT, 2><<<grid, kGroupThreads, 0, st>>>(p);
  else linear_groups_k<T, WIDE, G, MT, 3><<<grid, kGroupThreads, 0, st>>>(p);
  return launch_status();
}
// of a workgroup
static int most_rows(int x_type) { return x_type == MPQ_F32 ? 32 : 64; }
template <int T, bool WIDE, int G>
static int go_rows(const GroupsArgs& p, hipStream_t st) {
  constexpr int TERMS = Operand<T>::TERMS, SIZE = WIDE ? 4 : 2;
  const int64_t few = few_bytes(p.M, p.K, TERMS, G, SIZE);
  if (few <= 65536) {
    linear_groups_few_k<T, WIDE, G><<<(unsigned)((p.N + 15) / 16), kGroupThreads, (int)few, st>>>(p, (int)few - few_steps_bytes(p.K, G, SIZE));
    return launch_status();
  }
  if (p.M <= 16) return go<T, WIDE, G, 1>(p, st);
  if constexpr (T != MPQ_F32) {
    if (p.M > 32) return go<T, WIDE, G, 4>(p, st);
  }
  return go<T, WIDE, G, 2>(p, st);
}
template <int T, bool WIDE>
static int go_group(const GroupsArgs& p, int group, hipStream_t st) {
  return group == 32 ? go_rows<T, WIDE, 32>(p, st) : group == 64 ? go_rows<T, WIDE, 64>(p, st) : go_rows<T, WIDE, 128>(p, st);
}
template <int T>
static int go_type(const GroupsArgs& p, int group, hipStream_t st) {
  return p.scale_type == MPQ_F32 ? go_group<T, true>(p, group, st) : go_group<T, false>(p, group, st);
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
  const int64_t block = most_rows(x_type);
  if (N > (1 << 26) || (M + block - 1) / block > kMaxGridY) return MPQ_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(x) & (uintptr_t)(type_size(x_type) - 1)) return MPQ_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(w_scale) & (uintptr_t)(type_size(scale_type) - 1)) return MPQ_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(y_out) & (uintptr_t)(type_size(y_type) - 1)) return MPQ_ERR_ALIGN;
  if (M == 0) return MPQ_OK;
  if (!x || !w_q || !w_scale || !y_out) return MPQ_ERR_NULL;
  // an output where others still read
  const int x_el = (int)type_size(x_type), y_el = (int)type_size(y_type);
  const char* to = reinterpret_cast<const char*>(y_out);
  const int64_t to_bytes = M * N * y_el;
  auto meets = [&](const void* from, int64_t bytes) {
    const char* at = reinterpret_cast<const char*>(from);
    return to < at + bytes && at < to + to_bytes;
  };
  if (meets(w_q, N * (K / 2)) || meets(w_scale, N * (K / group) * (int64_t)type_size(scale_type))) return MPQ_ERR_SHAPE;
  if (meets(x, ((M - 1) * x_stride + K) * x_el)) {  // between two rows of x is no place of x
    const int64_t row = x_stride * x_el, behind = to - reinterpret_cast<const char*>(x);
    if (behind < 0 || behind % row < K * x_el || behind % row + to_bytes > row) return MPQ_ERR_SHAPE;
  }
  const GroupsArgs p{x, x_stride, w_q, w_scale, M, N, (int)K, scale_type, act, y_type, y_out};
  hipStream_t st = (hipStream_t)stream;
  if (x_type == MPQ_F32) return go_type<MPQ_F32>(p, group, st);
  return x_type == MPQ_BF16 ? go_type<MPQ_BF16>(p, group, st) : go_type<MPQ_F16>(p, group, st);
}
