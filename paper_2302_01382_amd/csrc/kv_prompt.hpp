// kv_prompt.hpp -- attention over quantized pages where a sequence brings many rows: a prompt's.
//
// The mathematics, the operands' order and the precision are kv_attention.hip's; there the codes' bytes count, here the
// matrix products do.  A wave takes NQ tiles of 16 rows of a key head (row, query head pairs: the heads of a group share keys
// and values), a workgroup its waves' rows.  Per step of 64 tokens the workgroup turns the codes of keys and
// values into fp16 once, on their way into a double-buffered LDS stage, and every wave multiplies them with its rows: an
// operand read out of the LDS serves NQ matrix steps.
//   keys    [token][chunk of 8 channels], chunks swizzled by the token so that 16 tokens' reads of one chunk fall into
//           different banks
//   values  [half step][quarter][channel][8 tokens]: the operand as a lane wants it, 16 lanes in 256 bytes
// A step's softmax: logits are at most one fused multiply-add from the product, f = row's scale * page's maximum, and
// their exponential takes the page's value factor along: P' = 2^(x - m + lg + 8), lg = log2 of the page's value maximum over
// a power of two that no maximum so far exceeds (at least -60); the sum divides it out again, page by page.  m is a maximum
// that may lag behind the true one by up to 6: P' then reaches 2^14, and the accumulators are rescaled only when it lags
// by more.
//
// Two prompts of up to 4500 rows behind up to 1000 tokens, 16 query and 4 key heads of 128 channels in bf16: 262 us, 868
// TFLOP/s of the pairs that the mask leaves.  Matrix steps take 35 % of the SIMDs' cycles, vector instructions (a third of them the
// exponentials, a quarter the codes' way into fp16) 55 %, with two waves per SIMD that 232 registers leave room for; a sixth of the
// time is the last workgroups' alone.  Operands are read out of the LDS four reads ahead, the first values' under the softmax (282
// with the compiler's one or two).  What did not help: the next keys' matrix steps between the exponentials (302 against
// 302), two groups of waves that take turns with matrix steps and softmax behind barriers (327 against 304), s_setprio around
// the matrix steps (302 to 307), 64 rows a wave (spilled).
#pragma once

#include "kv_attn.hpp"

#include <type_traits>

namespace mpq {

constexpr float kLag = 6.0f, kUp = 8.0f, kLeast = -60.0f, kMost = 1e30f;

// Maxima in assembly: the compiler's would first quiet every operand that it has not seen quieted.  Its hazard pass does not look into
// assembly, so that the waits around it are stated: results_ready between matrix steps and the maxima of their
// results, two states between a maximum and a swap of lanes.
__device__ __forceinline__ float max2(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// max over the four lanes that share a row: lane & 15
__device__ __forceinline__ float row_max(float v) {
  asm("s_nop 1" : "+v"(v));
  auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  v = max2(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
  asm("s_nop 1" : "+v"(v));
  auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  return max2(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}

// The results of matrix steps of four passes (16x16x32), for assembly to read: eight states behind the last of them.
template <int NQ>
__device__ __forceinline__ void results_ready(f32x4 (&sc)[2][NQ]) {
  static_assert(NQ <= 2, "all of them in one block: what comes behind it has waited");
  if constexpr (NQ == 1) asm volatile("s_nop 7" : "+v"(sc[0][0]), "+v"(sc[1][0]));
  else asm volatile("s_nop 7" : "+v"(sc[0][0]), "+v"(sc[1][0]), "+v"(sc[0][1]), "+v"(sc[1][1]));
}

// this wave's LDS accesses are done, and so are everyone's (loads from memory stay in flight)
__device__ __forceinline__ void lds_meet() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// SINGLE: one LDS stage, which leaves room for a third workgroup on a CU
template <int T, int DH, int NQ, bool SINGLE = false>
struct PromptCfg {
  // fp16 terms of q, and of a probability.  A second one of these takes a quarter of the time (bf16, two prompts of up to 4500 rows 262 |
  // 337 us).  It brings an fp16 output's distance to 64 bits from 3.0e-4 to 2.1e-4, its own rounding's.  A bf16 output's is 1.7e-3
  // either way: one term is off by 2^-11 at most, an eighth of bf16's half step, and outputs differ from those of fp32 products in one
  // step here and there (8.8e-4 of their power, 7.3e-5 with two).
  static constexpr int QT = T == MPQ_F32 ? 2 : 1, PT = T == MPQ_BF16 ? 1 : 2;
  // Waves: two workgroups of four share a CU, each at its own pace, and work comes in smaller pieces than with eight; dim > 128
  // fills the LDS with one workgroup (us, 8 | 4 waves: two prompts of up to 4500 rows of 16 / 4 heads of 128 306 | 283; 8 of 1000
  // of 12 heads of 64 60 | 42; 4096 rows of 32 / 8 heads of 128, no mask, where every piece is equal, 297 | 323; 4 of 300 of
  // 8 / 2 heads of 256 46.3 | 47.8).
  static constexpr int NW = DH == 4 ? 8 : 4, THREADS = NW * 64;
  static constexpr int ROWS = NW * 16 * NQ;                 // rows of a workgroup
  static constexpr int K_BYTES = 64 * DH * 128, STAGE = 2 * K_BYTES;
  static constexpr int LDS_BYTES = SINGLE ? STAGE : 2 * STAGE;
  static constexpr int NK = 256 * DH / THREADS, NV = NK;    // chunks per thread and step: 16 bytes of keys; twice 8 of values
};

// grid: pairs (sequence, head) fastest, a place further from one row tile to the next, so that each XCD has tiles of long and of
// short sequences; then splits; row tiles last, the last ones -- under a causal mask the longest -- first.
// ONE: a page holds at least a step's tokens, which then lie on one page.
// TREE: of a sequence's own rows, its last tokens, a row sees those that its bits name.  Its probabilities have both terms in every type: drafts
// are kept or dropped by what comes of them, and a call of few rows (kv_tree.hip) has both.
template <int T, int DH, int NQ, bool ONE, bool TREE, bool SINGLE = false>
__device__ __forceinline__ void prompt_rows_body(const AttnArgs& a, int64_t wg_tiles, const TreeMask& tree) {
  using C = PromptCfg<T, DH, NQ, SINGLE>;
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int QT = C::QT, PT = TREE ? 2 : C::PT, TT = 64;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, quarter = lane >> 4;
  const int64_t pairs = (int64_t)a.b.seqs * a.c.heads;
  const Digits at_grid = digits(pairs, a.splits, wg_tiles);
  if (at_grid.d[3] > 0) return;
  const int64_t g = at_grid.d[2];
  const int split = (int)at_grid.d[1];
  int64_t pair = at_grid.d[0] + (g - divide(g, pairs) * pairs);
  if (pair >= pairs) pair -= pairs;
  const int s = (int)divide(pair, a.c.heads), h = (int)(pair - (int64_t)s * a.c.heads);
  const Sequence sq = sequence(a.b, a.c.page, s);
  const int len = (int)(sq.len < sq.room ? sq.len : sq.room);  // (a length has 31 bits, and so has rows * group)
  const int64_t most = a.b.max_new < a.b.rows ? a.b.max_new : a.b.rows;  // (row_tiles, and 31 bits, were made for so many)
  const int before = (int)sq.len - sq.n, group = a.group, nrows = (int)(sq.n < most ? sq.n : most) * group;
  const int64_t row0_wide = (wg_tiles - 1 - g) * C::ROWS;
  if (row0_wide >= nrows) return;
  const int row0 = (int)row0_wide;
  const int D = a.c.dim;

  // tokens [lo, hi) that a row sees
  auto hi_of = [&](int row) {
    const int p = before + row / group;
    const int hi = a.causal && p < len ? p + 1 : len;
    return hi > 0 ? hi : 0;
  };
  auto lo_of = [&](int row) {
    const int64_t lo = a.window > 0 ? (int64_t)before + row / group - a.window + 1 : 0;
    return lo > 0 ? (int)(lo < 0x7FFFFFFF ? lo : 0x7FFFFFFF) : 0;
  };
  // of some row of the workgroup, and of every row of the wave
  const int end = row0 + C::ROWS < nrows ? row0 + C::ROWS : nrows;
  const int w0 = row0 + wave * 16 * NQ, w1 = w0 + 16 * NQ < nrows ? w0 + 16 * NQ : nrows;
  const int span_lo = lo_of(row0), span_hi = hi_of(end - 1);
  const int all_lo = lo_of(w1 - 1), all_hi = TREE ? (before < 0 ? 0 : before < len ? before : len) : hi_of(w0 < nrows ? w0 : 0);

  int lo[NQ], hi[NQ], tree_row[NQ];
  f16x8 q[QT][NQ][2 * DH];
  float row_scale[NQ];
  const float qmax = (float)((1 << (a.c.bits - 1)) - 1);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int idx = w0 + n * 16 + r;
    const bool real = idx < nrows;
    const int row_at = real ? idx : 0, i = row_at / group;
    lo[n] = lo_of(row_at);
    hi[n] = real ? hi_of(row_at) : 0;
    tree_row[n] = i;
    const El* row = reinterpret_cast<const El*>(a.q) + (sq.row0 + i) * a.q_ts + (int64_t)(h * group + row_at - i * group) * a.q_hs;
    f32x8 v[2 * DH];
    float m = 0.0f;
#pragma unroll
    for (int c = 0; c < 2 * DH; ++c) {
      const int d = c * 32 + quarter * 8;
      v[c] = real && d < D ? E::load8(row + d) : f32x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[c][e]));
    }
    m = row_max(m);
    const int e2 = 14 - (m > 0.0f ? __builtin_amdgcn_frexp_expf(m) : 0);
    const float sign = a.scale < 0.0f ? -1.0f : 1.0f;  // so that factors of products are never negative
#pragma unroll
    for (int c = 0; c < 2 * DH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __builtin_ldexpf(v[c][e] * sign, e2);
        const _Float16 top = (_Float16)x;
        q[0][n][c][e] = top;
        if (QT == 2) q[QT - 1][n][c][e] = (_Float16)(x - (float)top);
      }
    row_scale[n] = __builtin_ldexpf(fabsf(a.scale) * kLog2e / qmax, -e2);
  }

  // this workgroup's steps
  const int first = span_lo / TT, steps = span_hi > span_lo ? (span_hi + TT - 1) / TT - first : 0;
  const int per = (steps + a.splits - 1) / a.splits;
  const int t0 = first + split * per, t1 = first + ((split + 1) * per < steps ? (split + 1) * per : steps);
  const int32_t* table = a.b.table + (int64_t)s * a.b.table_pages;
  const unsigned page_bytes = (unsigned)(a.c.page * D);
  const int shift = 31 - __builtin_clz((unsigned)a.c.page), page_mask = a.c.page - 1;

  // Codes are requested one step ahead, the pages that they lie on looked up two steps ahead.  All through vector loads: a
  // scalar load in flight would make every wait for the LDS a wait for memory.  16 tokens lie on one page; where all 64
  // do, it is the same for every lane and addresses are a scalar base and the lane's constant offset.  Nothing here asks
  // whether it is needed: tokens that no row sees are looked up as the last one that some row does, chunks beyond dim are
  // fetched as the last one within (they meet zeros of q, or channels that are not stored), threads beyond the last chunk fetch
  // an earlier one again.
  constexpr int NP = ONE ? 1 : 4;  // pages of a step
  const unsigned pages = (unsigned)(a.c.pages < 0x7FFFFFFF ? a.c.pages : 0x7FFFFFFF);
  int k_token[C::NK], v_token[C::NV];        // of the thread's chunks: the first of the 16 tokens they belong to
  unsigned k_off[C::NK], v_off[C::NV];       // offset from there
#pragma unroll
  for (int j = 0; j < C::NK; ++j) {
    const int i = tid + j * C::THREADS, token = i / (4 * DH) & 63, d = i % (4 * DH) * 16;
    k_token[j] = token & ~15;
    k_off[j] = (unsigned)((token & 15) * D + (d < D ? d : D - 16));
  }
  // values: two channels of two groups of four tokens, 16 tokens apart; channels 0, 1 of four and 2, 3 go to different waves
#pragma unroll
  for (int j = 0; j < C::NV; ++j) {
    const int i = tid + j * C::THREADS, ksq = i / (16 * DH) & 7, d = i % (16 * DH) * 4 + (i / (128 * DH) & 1) * 2;
    v_token[j] = (ksq >> 2) * 32;
    v_off[j] = (unsigned)(((ksq & 3) * D + (d < D ? d : D - 2)) * 4);
  }
  int idk[C::NK], idv[C::NV][2], idu;
  auto look_up = [&](int t) {
    auto page = [&](int place) {
      const int tok = t * TT + place;  // (at most a few steps past kMostTokens)
      int at = (tok < span_hi ? tok : span_hi - 1) >> shift;
      asm volatile("" : "+v"(at));
      return table[at];
    };
    if (!ONE) {
#pragma unroll
      for (int j = 0; j < C::NK; ++j) idk[j] = page(k_token[j]);
#pragma unroll
      for (int j = 0; j < C::NV; ++j) {
        idv[j][0] = page(v_token[j]);
        idv[j][1] = page(v_token[j] + 16);
      }
    }
    idu = page(ONE ? 0 : (lane & 3) * 16);
  };
  bool page_ok;
  float mk_in, mv_in;  // lane u (mod 4): maxima of the pages of tokens 16 u .. of the step that is in flight
  v4i kw[C::NK];
  v2i vw[C::NV][2];
  auto request = [&](int t) {
    page_ok = (unsigned)idu < pages;
    uint64_t at = (uint64_t)(page_ok ? (unsigned)idu : 0u) * (unsigned)a.c.heads + (unsigned)h;
    mk_in = a.c.k_absmax[at];
    mv_in = a.c.v_absmax[at];
    if (ONE) {
      const uint64_t id = (unsigned)__builtin_amdgcn_readfirstlane(page_ok ? idu : 0);
      const uint64_t first_byte = (id * (unsigned)a.c.heads + (unsigned)h) * page_bytes + (unsigned)(((t * TT) & page_mask) * D);
      const int8_t *kp = a.c.k_codes + first_byte, *vp = a.c.v_codes + first_byte;
#pragma unroll
      for (int j = 0; j < C::NK; ++j) kw[j] = *reinterpret_cast<const v4i*>(kp + (unsigned)(k_off[j] + k_token[j] * D));
#pragma unroll
      for (int j = 0; j < C::NV; ++j) {
        vw[j][0] = *reinterpret_cast<const v2i*>(vp + (unsigned)(v_off[j] + v_token[j] * D));
        vw[j][1] = *reinterpret_cast<const v2i*>(vp + (unsigned)(v_off[j] + (v_token[j] + 16) * D));
      }
    } else {
      auto at_page = [&](const int8_t* codes, int id, int token, unsigned off) {
        const uint64_t page = (uint64_t)((unsigned)id < pages ? (unsigned)id : 0u) * (unsigned)a.c.heads + (unsigned)h;
        return codes + page * page_bytes + ((unsigned)(((t * TT + token) & page_mask) * D) + off);
      };
#pragma unroll
      for (int j = 0; j < C::NK; ++j) kw[j] = *reinterpret_cast<const v4i*>(at_page(a.c.k_codes, idk[j], k_token[j], k_off[j]));
#pragma unroll
      for (int j = 0; j < C::NV; ++j) {
        vw[j][0] = *reinterpret_cast<const v2i*>(at_page(a.c.v_codes, idv[j][0], v_token[j], v_off[j]));
        vw[j][1] = *reinterpret_cast<const v2i*>(at_page(a.c.v_codes, idv[j][1], v_token[j] + 16, v_off[j]));
      }
    }
  };
  auto store = [&](unsigned stage) {
#pragma unroll
    for (int j = 0; j < C::NK; ++j) {
      const int i = tid + j * C::THREADS, token = i / (4 * DH) & 63, ch = i % (4 * DH) * 2;
      const int swz = DH == 1 ? (token >> 1) & 7 : token & 15;
      char* row = lds + stage + token * (DH * 128);
      *reinterpret_cast<f16x8*>(row + ((ch ^ swz) << 4)) = codes8(kw[j].x, kw[j].y);
      *reinterpret_cast<f16x8*>(row + (((ch ^ swz) << 4) ^ 16)) = codes8(kw[j].z, kw[j].w);
    }
#pragma unroll
    for (int j = 0; j < C::NV; ++j) {
      const int i = tid + j * C::THREADS, ksq = i / (16 * DH) & 7, dq = i % (16 * DH), two = i / (128 * DH) & 1;
      char* to = lds + stage + C::K_BYTES + ((ksq * 64 * DH + (dq >> 4) * 64 + (dq & 15)) << 4) + two * 512;
#pragma unroll
      for (int k = 0; k < 2; ++k) *reinterpret_cast<f16x8*>(to + k * 256) = codes8(vw[j][0][k], vw[j][1][k]);
    }
  };

  // m: what exponentials of the row refer to (0 before its first visible token); the maximum may pass it by kLag, up to top
  float m_use[NQ], m_top[NQ], l_run[NQ];
  int v_exp = -100000;  // O' is in units of 2^(v_exp - 8)
  f32x4 o[NQ][4 * DH];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_use[n] = 0.0f;
    m_top[n] = -__builtin_inff();
    l_run[n] = 0.0f;
#pragma unroll
    for (int k = 0; k < 4 * DH; ++k) o[n][k] = f32x4{0, 0, 0, 0};
  }

  if (t0 < t1) {
    look_up(t0);
    request(t0);
    look_up(t0 + 1);
    store(0);
  }
  // Of the pages of a step: keys' maximum (negative: no such page), log2 of the values' factor + 8 and the factor's
  // reciprocal; v_next: exponent of the power of two that the factors refer to.
  float mk[NP], lg[NP], back[NP];
  int v_next = v_exp;
  auto arrived = [&]() {
    mk_in = page_ok ? mk_in : -1.0f;
    const bool any = page_ok && mv_in > 0.0f;
    // (a maximum of infinity moves no exponent and gives a factor whose sum with minus infinity is minus infinity: rows that see
    // the page become NaN, rows that do not see it keep their value)
    int e = any && mv_in < __builtin_inff() ? __builtin_amdgcn_frexp_expf(mv_in) : v_next;
    if (!ONE) {
      e = max(e, __builtin_amdgcn_update_dpp(0, e, kQuadSwap1, 0xF, 0xF, true));
      e = max(e, __builtin_amdgcn_update_dpp(0, e, kQuadSwap2, 0xF, 0xF, true));
    }
    e = __builtin_amdgcn_readfirstlane(e);
    v_next = e > v_next ? e : v_next;
    // (a page of maximum 0 as one of the least factor: its probabilities vanish in fp16, 2^(kLag + kUp + kLeast) at most, and
    // count in the sum)
    const float l2 = any ? fminf(fmaxf(__builtin_amdgcn_logf(__builtin_ldexpf(mv_in, -v_next)), kLeast), kMost) : kLeast;
    const float inverse = __builtin_amdgcn_exp2f(-l2);
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      mk[u] = f_from_bits(__builtin_amdgcn_readlane(bits_from_f(mk_in), u));
      lg[u] = f_from_bits(__builtin_amdgcn_readlane(bits_from_f(l2 + kUp), u));
      back[u] = f_from_bits(__builtin_amdgcn_readlane(bits_from_f(inverse), u));
    }
  };
  if (t0 < t1) arrived();
  lds_meet();
  const unsigned k_at = (unsigned)(r * (DH * 128)), v_at = (unsigned)(C::K_BYTES + ((quarter * 64 * DH + r) << 4));
  const unsigned swz = (unsigned)(DH == 1 ? (r >> 1) & 7 : r);
  unsigned stage = 0;
  for (int t = t0; t < t1; ++t) {
    const bool more = t + 1 < t1;
    if (more) {
      request(t + 1);
      look_up(t + 2);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // 32 tokens at a time
      const int base = t * TT + half * 32;
      f32x4 sc[2][NQ];
      // reads are issued so many ahead of the matrix steps that take them
      constexpr int NR = 4 * DH, kAhead = 4;
      auto read_k = [&](int i) {
        const int c = i >> 1, u = i & 1;
        return *reinterpret_cast<const f16x8*>(lds + stage + k_at + (((unsigned)(4 * c + quarter) ^ swz) << 4) + (2 * half + u) * 16 * (DH * 128));
      };
      auto read_v = [&](int k) { return *reinterpret_cast<const f16x8*>(lds + stage + v_at + ((half * 4 * 64 * DH + k * 16) << 4)); };
      f16x8 kf[kAhead], vf[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = read_k(i);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NQ; ++n) sc[u][n] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        const f16x8 now = kf[i % kAhead];
#pragma unroll
        for (int x = 0; x < QT; ++x)
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            sc[i & 1][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now, q[x][n][i >> 1], sc[i & 1][n], 0, 0, 0);
        if (i + kAhead < NR) kf[i % kAhead] = read_k(i + kAhead);
        else vf[i + kAhead - NR] = read_v(i + kAhead - NR);
      }
      __builtin_amdgcn_sched_barrier(0);
      results_ready<NQ>(sc);
      // logits over f; scalars: see kv_attention.hip
      float x[2][NQ][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[u][n][e] = sc[u][n][e];
      const float mk0 = mk[ONE ? 0 : 2 * half], mk1 = mk[ONE ? 0 : 2 * half + 1];
      if (mk0 < 0.0f || mk1 < 0.0f || base < all_lo || base + 32 > all_hi) {  // uniform over the wave
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          const int from = lo[n] - base - quarter * 4, to = hi[n] - base - quarter * 4;  // counted from the lane's first token
          // (TREE) the lane's first token is bit 0, the one 16 u + e behind it bit 16 u + e
          const uint64_t bits = TREE ? tree_bits(tree, sq.row0 + tree_row[n], (int64_t)base + quarter * 4 - before) : 0;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool out = (16 * u + e < from) | (16 * u + e >= to) | ((u ? mk1 : mk0) < 0.0f) | (TREE && !(bits >> (16 * u + e) & 1));
              x[u][n][e] = out ? -__builtin_inff() : x[u][n][e];
            }
        }
      }
      // f: at least 1e-30, so that it leaves an infinity one (a smaller one means a logit of 0 either way).  A row's maximum
      // passes the limit where that of one of its four lanes does.
      float f[2][NQ], top[NQ];
      bool grow = v_next != v_exp;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        f[0][n] = max2(row_scale[n] * mk0, 1e-30f);
        const float a0 = max2(max3(x[0][n][0], x[0][n][1], x[0][n][2]), x[0][n][3]);
        if (ONE) {
          f[1][n] = f[0][n];
          top[n] = max3(max3(a0, x[1][n][0], x[1][n][1]), x[1][n][2], x[1][n][3]) * f[0][n];
        } else {
          f[1][n] = max2(row_scale[n] * mk1, 1e-30f);
          const float a1 = max2(max3(x[1][n][0], x[1][n][1], x[1][n][2]), x[1][n][3]);
          top[n] = max2(a0 * f[0][n], a1 * f[1][n]);
        }
        grow |= top[n] > m_top[n];
      }
      if (__any(grow)) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          const float m_old = m_top[n] == -__builtin_inff() ? m_top[n] : m_use[n], m_new = max2(row_max(top[n]), m_old);
          m_use[n] = m_new == -__builtin_inff() ? 0.0f : m_new;
          m_top[n] = m_new + kLag;
          const float alpha = __builtin_amdgcn_exp2f(m_old - m_use[n]);
          l_run[n] *= alpha;
          const float scale = __builtin_ldexpf(alpha, v_exp - v_next);
#pragma unroll
          for (int k = 0; k < 4 * DH; ++k) o[n][k] *= scale;
        }
        v_exp = v_next;
      }
      float half_sum[NQ];
      v4i pw[PT][NQ];  // probabilities: eight fp16, as the value product wants them
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          __builtin_amdgcn_sched_barrier(0);
          const int pg = ONE ? 0 : 2 * half + u;
          const float mm = lg[pg] - m_use[n];
          float w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][n][e], f[u][n], mm));
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const f16x2 top16 = __builtin_convertvector(f32x2{w[e], w[e + 1]}, f16x2);
            pw[0][n][u * 2 + e / 2] = __builtin_bit_cast(int, top16);
            if (PT == 2)
              pw[PT - 1][n][u * 2 + e / 2] =
                  __builtin_bit_cast(int, __builtin_convertvector(f32x2{w[e] - (float)top16.x, w[e + 1] - (float)top16.y}, f16x2));
          }
          const float sum = (w[0] + w[1]) + (w[2] + w[3]);
          if (!ONE) l_run[n] = __builtin_fmaf(sum, back[pg], l_run[n]);
          else if (u == 0) half_sum[n] = sum;
          else l_run[n] = __builtin_fmaf(half_sum[n] + sum, back[0], l_run[n]);
        }
      }
#pragma unroll
      for (int k = 0; k < 4 * DH; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        const f16x8 now = vf[k % kAhead];
#pragma unroll
        for (int x = 0; x < PT; ++x)
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            o[n][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now, __builtin_bit_cast(f16x8, pw[x][n]), o[n][k], 0, 0, 0);
        if (k + kAhead < NR) vf[k % kAhead] = read_v(k + kAhead);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (SINGLE) lds_meet();
    else stage = (unsigned)C::STAGE - stage;
    if (more) store(stage);
    if (more) arrived();
    lds_meet();
  }

  // lane (row r, quarter): channels 64 c + 16 quarter + 4 e + k in o[n][4 c + k][e]
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float l = l_run[n];
    l += across(l, 16);
    l += across(l, 32);
    const int at = w0 + n * 16 + r;
    if (at >= nrows) continue;
    const float f = l == 0.0f ? 0.0f : 1.0f / qmax * (a.splits > 1 ? __builtin_amdgcn_exp2f(-kUp) : 1.0f / l);
    const int64_t slot = (pair * a.row_tiles + (at >> 4)) * a.splits + split;
    float* part = a.part_o + (slot * 16 + r) * D;
    const int i = at / group;
    El* to = reinterpret_cast<El*>(a.out) + (sq.row0 + i) * a.o_ts + (int64_t)(h * group + at - i * group) * a.o_hs;
#pragma unroll
    for (int c = 0; c < DH; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = c * 64 + quarter * 16 + 4 * e;
        if (d >= D) continue;
        const f32x4 v = f32x4{o[n][4 * c][e], o[n][4 * c + 1][e], o[n][4 * c + 2][e], o[n][4 * c + 3][e]} * f;
        if (a.splits > 1) *reinterpret_cast<f32x4*>(part + d) = v;
        else E::store4(to + d, times_two_to(v, v_exp));
      }
    if (a.splits > 1 && quarter == 0)
      a.part[slot * 16 + r] = Partial{m_top[n] == -__builtin_inff() ? m_top[n] : m_use[n], l * __builtin_amdgcn_exp2f(-kUp), (float)v_exp};
  }
}

// K: the kernels, and what they take besides the call and its tiles
template <typename K, int T, int DH, int NQ>
static int prompt_go(const K& k, const AttnArgs& a, int64_t wg_tiles, bool prepare_only, hipStream_t st) {
  using C = typename K::template Cfg<T, DH, NQ>;
  using Kern = typename K::Kern;
  static const Kern kerns[2] = {K::template kernel<T, DH, NQ, false>(), K::template kernel<T, DH, NQ, true>()};
  static std::atomic<unsigned> done[kMaxDevices];
  for (int one = 0; one < 2; ++one) {
    if (C::LDS_BYTES <= 65536 || (!prepare_only && one != (a.c.page >= 64))) continue;
    const int rc = allow_lds(reinterpret_cast<const void*>(kerns[one]), C::LDS_BYTES, done, one);
    if (rc != MPQ_OK) return rc;
  }
  if (prepare_only) return MPQ_OK;
  const dim3 grid = wide_grid(wg_tiles * a.splits * a.b.seqs * a.c.heads, C::THREADS);
  return k.launch(kerns[a.c.page >= 64], grid, C::THREADS, C::LDS_BYTES, st, a, wg_tiles);
}

template <typename K, int T>
static int prompt_go_type(const K& k, const AttnArgs& a, int64_t wg_tiles, int wg_rows, bool prepare_only, hipStream_t st) {
  constexpr int WIDE = T == MPQ_F32 ? 1 : 2;
  if (a.c.dim > 128) return prompt_go<K, T, 4, 1>(k, a, wg_tiles, prepare_only, st);
  if (a.c.dim > 64) return wg_rows == 64 ? prompt_go<K, T, 2, 1>(k, a, wg_tiles, prepare_only, st) : prompt_go<K, T, 2, WIDE>(k, a, wg_tiles, prepare_only, st);
  return wg_rows == 64 ? prompt_go<K, T, 1, 1>(k, a, wg_tiles, prepare_only, st) : prompt_go<K, T, 1, 2>(k, a, wg_tiles, prepare_only, st);
}

template <typename K>
static int prompt_launch(const K& k, int type, const AttnArgs& a, int64_t wg_tiles, int wg_rows, bool prepare_only, hipStream_t st) {
  if (type == MPQ_F32) return prompt_go_type<K, MPQ_F32>(k, a, wg_tiles, wg_rows, prepare_only, st);
  if (type == MPQ_BF16) return prompt_go_type<K, MPQ_BF16>(k, a, wg_tiles, wg_rows, prepare_only, st);
  return prompt_go_type<K, MPQ_F16>(k, a, wg_tiles, wg_rows, prepare_only, st);
}

// allows the kernels the LDS they need on the current device
template <typename K>
static int prompt_prepare() {
  for (int type : {MPQ_F32, MPQ_BF16, MPQ_F16})
    for (int dim : {64, 128, 256})
      for (int rows : {64, 128}) {
        AttnArgs a{};
        a.c.dim = dim;
        const int rc = prompt_launch(K{}, type, a, 0, rows, true, nullptr);
        if (rc != MPQ_OK) return rc;
      }
  return MPQ_OK;
}

}  // namespace mpq
