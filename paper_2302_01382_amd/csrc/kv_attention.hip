// kv_attention.hip -- attention over a cache of quantized pages.
//
// For a row q at position p of its sequence and a key head:  o = sum_j P_j V_j, P = softmax_j(c q . K_j) over the visible
// tokens j, K_j = code * (m_k / qmax) and V_j likewise with ONE maximum per page and head.  So both products run on the
// codes themselves, which fp16 holds exactly, and a page's maximum is a factor of its 16 tokens' logits (keys) or
// probabilities (values).
//
// One pass over the tokens with the running maximum and sum of the softmax, in registers alone:
//   S' = K q'     16 tokens x 16 rows:  a lane holds four tokens of one row (lane & 15)
//   O' = V' P'    16 channels x 16 rows: the operand P' of v_mfma_f32_16x16x32_f16 wants, from that same lane, eight tokens of
//                 that row -- four of each of two S' tiles, which is what it holds.  The other operand is then four tokens of
//                 a channel from each of the two tiles: a dword of the cache's value order [page / 4][dim][4] each.
// No LDS, no transposition; the order of k within a product is free.
//
// Precision: logits, maxima, sums and outputs are fp32.  q goes in as fp16 after a scaling by a power of two (its row's
// largest entry to 2^14: bf16 and fp16 keep every bit down to 2^-28 of that entry), fp32 as two such terms (22 bits).
// Probabilities, at most 1, go in as fp16 times 2^14, as two such terms: with one, an fp16 output's distance to 64 bits went from
// 2.1e-4 to 3.1e-4, and a bf16 one, whose distance stays at 1.7e-3, differed from the output of fp32 products by 8.9e-4 of its power
// instead of 6.3e-5 (64 sequences of up to 8192 tokens 151.3 -> 152.4 us with the second term).
// Values' maxima differ from page to page: probabilities carry them relative to a power of two that is at least the largest
// maximum so far, an exact rescaling whenever it grows.
#include "kv_attn.hpp"

namespace mpq {

__device__ __forceinline__ v4i stream16(const int8_t* p) {
  return __builtin_nontemporal_load((const __attribute__((address_space(1))) v4i*)p);
}
constexpr int kPBits = 14;  // probabilities are multiplied by 2^14 before they are rounded to fp16

template <int T, int DH>
struct AttnShape {
  static constexpr int QT = T == MPQ_F32 ? 2 : 1;   // fp16 terms of q
  static constexpr int TT = DH <= 2 ? 64 : 32;  // tokens per step
  static constexpr int NS = TT / 16;
  static constexpr int DP = DH * 64;
};

// grid: ((sequence * heads + head) * row_tiles + tile) * splits + split.  DH: dim in units of 64, rounded up.
// ONE: a page holds at least a step's tokens, which then lie on one page.  NW: waves.
template <int T, int DH, bool ONE, int NW>
__global__ __launch_bounds__(NW * 64) void kv_attention_k(AttnArgs a) {
  using S = AttnShape<T, DH>;
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int QT = S::QT, TT = S::TT, NS = S::NS, DP = S::DP, NP = ONE ? 1 : NS;
  __shared__ float sm_m[NW][16], sm_l[NW][16];
  __shared__ int sm_e[NW];
  __shared__ __attribute__((aligned(16))) float sm_o[NW / 2][16][DP + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, quarter = lane >> 4;
  const Digits g = digits(a.splits, a.row_tiles, a.c.heads);
  const int split = (int)g.d[0], h = (int)g.d[2];
  const int64_t slot = block_index(), tile = g.d[1], s = g.d[3];  // slot: of the partial results
  if (s >= a.b.seqs) return;
  const Sequence sq = sequence(a.b, a.c.page, (int)s);
  const int64_t len = sq.len < sq.room ? sq.len : sq.room;
  const int64_t nrows = (int64_t)sq.n * a.group;
  if (tile * 16 >= nrows) return;
  const int D = a.c.dim;

  // this lane's row: its position, what it sees
  const unsigned group = (unsigned)a.group, row0 = (unsigned)(tile * 16), idx = row0 + (unsigned)r;  // (32 bits: row_tiles)
  const bool real = idx < nrows;
  const int64_t i = real ? idx / group : 0;
  const int qh = h * a.group + (real ? (int)(idx - (unsigned)i * group) : 0);
  auto row_sees = [&](int64_t row) { return seen(sq.len - sq.n + row, len, a.causal, a.window); };
  const Span own = row_sees(i);
  const int64_t lo = own.lo, hi = real ? own.hi : 0;
  // of the whole tile: its first and last token row, what some row of it sees, and what every row does, which needs no mask
  const int64_t first_row = row0 / group, last_row = (row0 + 15 < nrows ? row0 + 15 : (unsigned)(nrows - 1)) / group;
  const Span of_first = row_sees(first_row), of_last = row_sees(last_row), span = {of_first.lo, of_last.hi};
  const int64_t all_lo = of_last.lo, all_hi = of_first.hi;

  // q: lane (row, quarter) holds channels 64 c + 16 quarter .. + 15 for every c, as the keys come
  f16x8 q[QT][2 * DH];
  float row_scale;
  {
    const El* row = reinterpret_cast<const El*>(a.q) + (sq.row0 + i) * a.q_ts + (int64_t)qh * a.q_hs;
    f32x8 v[2 * DH];
    float m = 0.0f;
#pragma unroll
    for (int c = 0; c < 2 * DH; ++c) {
      const int d = (c >> 1) * 64 + quarter * 16 + (c & 1) * 8;
      v[c] = real && d < D ? E::load8(row + d) : f32x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[c][e]));
    }
    m = fmaxf(m, across(m, 16));
    m = fmaxf(m, across(m, 32));
    const int e2 = kPBits - (m > 0.0f ? __builtin_amdgcn_frexp_expf(m) : 0);
#pragma unroll
    for (int c = 0; c < 2 * DH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __builtin_ldexpf(v[c][e], e2);
        const _Float16 top = (_Float16)x;
        q[0][c][e] = top;
        if (QT == 2) q[QT - 1][c][e] = (_Float16)(x - (float)top);
      }
    // logits in units of log 2
    const float qmax = (float)((1 << (a.c.bits - 1)) - 1);
    row_scale = __builtin_ldexpf(a.scale * kLog2e / qmax, -e2);
  }

  // this workgroup's tokens: whole steps, dealt out to the splits in one piece each and to the waves in turn
  const Steps share = steps_of(span, TT, a.splits, split);
  const int64_t t0 = share.t0, t1 = share.t1;
  const int32_t* table = a.b.table + s * a.b.table_pages;
  const int64_t page_bytes = (int64_t)a.c.page * D;
  const int shift = 31 - __builtin_clz((unsigned)a.c.page);

  // What a step needs of its tokens, by page: NP pages of TT / NP tokens each.  Pages are looked up a step ahead of the
  // codes they hold, codes are requested a step ahead of the products.
  int id[NP];
  auto look_up = [&](int64_t t) {
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int64_t tok = t * TT + u * (TT / NP);
      id[u] = t < t1 && tok < span.hi ? table[tok >> shift] : -1;
    }
  };
  const int8_t *kp[NP], *vp[NP];
  float mk[NP], mv[NP];
  auto locate = [&](int64_t t) {
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const bool ok = id[u] >= 0 && id[u] < a.c.pages;
      const int64_t at = (int64_t)(ok ? id[u] : 0) * a.c.heads + h;
      const int place = (int)((t * TT + u * (TT / NP)) & (a.c.page - 1));
      kp[u] = a.c.k_codes + at * page_bytes + place * D;
      vp[u] = a.c.v_codes + at * page_bytes + place * D;
      mk[u] = ok ? a.c.k_absmax[at] : -1.0f;
      mv[u] = ok ? a.c.v_absmax[at] : 0.0f;
    }
  };
  v4i kw[NS][DH], vw[NS][DH];
  auto request_k = [&]() {
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
      for (int c = 0; c < DH; ++c) {
        const int d = c * 64 + quarter * 16;
        kw[u][c] = d < D ? stream16(kp[u / (NS / NP)] + (u % (NS / NP) * 16 + r) * D + d) : v4i{0, 0, 0, 0};
      }
  };
  auto request_v = [&]() {
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
      for (int c = 0; c < DH; ++c) {
        const int d = c * 64 + r * 4;
        vw[u][c] = d < D ? stream16(vp[u / (NS / NP)] + u % (NS / NP) * 16 * D + (quarter * D + d) * 4) : v4i{0, 0, 0, 0};
      }
  };

  float m_run = -__builtin_inff(), l_run = 0.0f;
  int v_exp = -100000;  // O' is in units of 2^(v_exp - kPBits)
  f32x4 o[DH][4];
#pragma unroll
  for (int c = 0; c < DH; ++c)
#pragma unroll
    for (int k = 0; k < 4; ++k) o[c][k] = f32x4{0, 0, 0, 0};

  int64_t t = t0 + wave;
  if (t < t1) {
    look_up(t);
    locate(t);
    request_k();
    request_v();
    look_up(t + NW);
  }
  for (; t < t1; t += NW) {
    const int64_t base = t * TT;
    const bool more = t + NW < t1;
    // S': tokens 16 u + 4 quarter .. + 3 of the step, row r
    f32x4 sc[NS];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      sc[u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < DH; ++c) {
        const f16x8 k0 = codes8(kw[u][c].x, kw[u][c].y), k1 = codes8(kw[u][c].z, kw[u][c].w);
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[x][2 * c], sc[u], 0, 0, 0);
          sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[x][2 * c + 1], sc[u], 0, 0, 0);
        }
      }
    }
    float mk_now[NP], mv_now[NP];
    bool bad = false;
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      mk_now[u] = mk[u];
      mv_now[u] = mv[u];
      bad |= mk[u] < 0.0f;
    }
    if (more) {
      locate(t + NW);
      request_k();
      look_up(t + 2 * NW);
    }
    // logits, in scalars: where elements of the accumulator vectors themselves were overwritten under a lane's condition, the
    // compiler (hipcc 7.2) spread the first one's value over the three others
    float x[NS][4];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      const float f = row_scale * mk_now[u / (NS / NP)];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = sc[u][e] * f;
    }
    if (bad || base < all_lo || base + TT > all_hi) {  // uniform
      // the row's first and last visible token, counted from the lane's first of the step
      const int64_t at = base + quarter * 4;
      const int from = (int)(lo - at < -1 ? -1 : lo - at > TT ? TT : lo - at), to = (int)(hi - at < -TT ? -TT : hi - at > TT ? TT : hi - at);
#pragma unroll
      for (int u = 0; u < NS; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool out = (16 * u + e < from) | (16 * u + e >= to) | (mk_now[u / (NS / NP)] < 0.0f);
          x[u][e] = out ? -__builtin_inff() : x[u][e];
        }
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, x[u][e]);
    top = fmaxf(top, across(top, 16));
    top = fmaxf(top, across(top, 32));
    int ve = v_exp;
#pragma unroll
    for (int u = 0; u < NP; ++u)
      if (mv_now[u] > 0.0f && mv_now[u] < __builtin_inff()) {
        const int e = __builtin_amdgcn_frexp_expf(mv_now[u]);
        ve = e > ve ? e : ve;
      }
    const float m_new = fmaxf(m_run, top);
    const float m_use = m_new == -__builtin_inff() ? 0.0f : m_new;
    if (ve != v_exp || __any(m_new > m_run)) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      l_run *= alpha;
      const float f = __builtin_ldexpf(alpha, v_exp - ve);
#pragma unroll
      for (int c = 0; c < DH; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[c][k] *= f;
      v_exp = ve;
      m_run = m_new;
    }
    f16x4 p[2][NS];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      // (a maximum of infinity as a factor that leaves a probability of 0 one: rows that see the page become NaN, others do not)
      const float v = mv_now[u / (NS / NP)], f = v > 0.0f ? fminf(__builtin_ldexpf(v, kPBits - v_exp), __FLT_MAX__) : 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float w = __builtin_amdgcn_exp2f(x[u][e] - m_use);
        l_run += w;
        float y = w * f;
        // its fp32 rounding stays: the product and its conversion would become one instruction that rounds once, the difference
        // below would be to another fp16 value, and one probability in a thousand off by 2^-10
        asm("" : "+v"(y));
        const _Float16 hi16 = (_Float16)y;
        p[0][u][e] = hi16;
        p[1][u][e] = (_Float16)(y - (float)hi16);
      }
    }
    // O': channels 64 c + 4 (lane & 15) + k of the value operand
#pragma unroll
    for (int u = 0; u < NS; u += 2) {
#pragma unroll
      for (int c = 0; c < DH; ++c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f16x8 v = codes8(vw[u][c][k], vw[u + 1][c][k]);
#pragma unroll
          for (int term = 0; term < 2; ++term) {
            const f16x8 pp = __builtin_shufflevector(p[term][u], p[term][u + 1], 0, 1, 2, 3, 4, 5, 6, 7);
            o[c][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pp, o[c][k], 0, 0, 0);
          }
        }
      }
    }
    if (more) request_v();
  }
  // a row's sum over its four lanes; the waves' shares joined: a lane holds, of row r, channels
  // 64 c + 16 quarter + 4 e + k in o[c][k][e]
  l_run += across(l_run, 16);
  l_run += across(l_run, 32);
  if (quarter == 0) {
    sm_m[wave][r] = m_run;
    sm_l[wave][r] = l_run;
  }
  if (lane == 0) sm_e[wave] = v_exp;
  __syncthreads();
  float m_all = sm_m[0][r];
  int e_all = sm_e[0];  // shares are added in units of 2^e_all: they are as large as the sum then, whatever the values are
#pragma unroll
  for (int w = 1; w < NW; ++w) {
    m_all = fmaxf(m_all, sm_m[w][r]);
    e_all = max(e_all, sm_e[w]);
  }
  const float m_use = m_all == -__builtin_inff() ? 0.0f : m_all;
  const float mine = __builtin_amdgcn_exp2f(m_run - m_use);
  const float qmax = (float)((1 << (a.c.bits - 1)) - 1);
  const float f = l_run > 0.0f ? __builtin_ldexpf(mine / qmax, v_exp - e_all - kPBits) : 0.0f;
#pragma unroll
  for (int half = 1; half >= 0; --half) {  // the upper half of the waves leaves its share, the lower half adds its own
    if (wave / (NW / 2) == half) {
#pragma unroll
      for (int c = 0; c < DH; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x4* to = reinterpret_cast<f32x4*>(&sm_o[wave % (NW / 2)][r][c * 64 + quarter * 16 + 4 * e]);
          const f32x4 v = f32x4{o[c][0][e], o[c][1][e], o[c][2][e], o[c][3][e]} * f;
          *to = half ? v : v + *to;
        }
    }
    __syncthreads();
  }
  for (int x = threadIdx.x; x < 16 * (D >> 2); x += NW * 64) {
    const int row = x / (D >> 2), d = (x % (D >> 2)) * 4;
    float top = sm_m[0][row];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, sm_m[w][row]);
    const float use = top == -__builtin_inff() ? 0.0f : top;
    float l = 0.0f;
    f32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w) l += sm_l[w][row] * __builtin_amdgcn_exp2f(sm_m[w][row] - use);
#pragma unroll
    for (int w = 0; w < NW / 2; ++w) v += *reinterpret_cast<const f32x4*>(&sm_o[w][row][d]);
    const int64_t at = tile * 16 + row;
    if (at >= nrows) continue;
    if (a.splits > 1) {
      *reinterpret_cast<f32x4*>(a.part_o + (slot * 16 + row) * D + d) = v;
      if (d == 0) a.part[slot * 16 + row] = Partial{top, l, (float)e_all};
      continue;
    }
    const unsigned token = (unsigned)at / group;
    El* to = reinterpret_cast<El*>(a.out) + (sq.row0 + token) * a.o_ts + (int64_t)(h * a.group + (int)((unsigned)at - token * group)) * a.o_hs + d;
    E::store4(to, l == 0.0f ? f32x4{0, 0, 0, 0} : times_two_to(v / l, e_all));  // (a row with a NaN in q has one in l)
  }
}

// Joins the splits of a row: a workgroup per row, its threads over groups of four channels and, as many as are left, over
// the splits.  (A workgroup per 16 rows, each thread over all splits: 51 us for 8 tiles of 96 splits of 128 channels.)
// grid: ((sequence * heads + head) * row_tiles + tile) * tile_rows + row.
template <int T>
__global__ __launch_bounds__(kBlock) void kv_attention_join_k(AttnArgs a) {
  using E = Elem<T>;
  typedef typename E::type El;
  __shared__ __attribute__((aligned(16))) float sm_o[kBlock * 4];
  __shared__ float sm_l[kBlock], sm_m[kBlock / kWave], sm_e[kBlock / kWave];
  const Digits g = digits(a.tile_rows, a.row_tiles, a.c.heads);
  const int row = (int)g.d[0], h = (int)g.d[2];
  const int64_t tile = g.d[1], s = g.d[3], slot = ((s * a.c.heads + h) * a.row_tiles + tile) * a.splits;
  if (s >= a.b.seqs) return;
  const Sequence sq = sequence(a.b, a.c.page, (int)s);
  const int64_t at = tile * 16 + row;
  if (at >= joined_rows(a, sq)) return;
  const int D = a.c.dim, quads = D >> 2, parts = kBlock / quads;
  const int d = ((int)threadIdx.x % quads) * 4, part = (int)threadIdx.x / quads;
  const Partial* of = a.part + slot * 16 + row;  // the row's in the first split; 16 to the next
  float top = -__builtin_inff(), exponent = -__builtin_inff();
  for (int i = threadIdx.x; i < a.splits; i += kBlock) {
    const Partial x = of[(int64_t)i * 16];
    top = fmaxf(top, x.m);
    exponent = fmaxf(exponent, x.e);
  }
  top = wave_max(top);
  exponent = wave_max(exponent);
  if ((threadIdx.x & 63) == 0) {
    sm_m[threadIdx.x >> 6] = top;
    sm_e[threadIdx.x >> 6] = exponent;
  }
  __syncthreads();
  top = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
  const int e_all = (int)fmaxf(fmaxf(sm_e[0], sm_e[1]), fmaxf(sm_e[2], sm_e[3]));
  const float use = top == -__builtin_inff() ? 0.0f : top;
  float l = 0.0f;
  f32x4 v = {0, 0, 0, 0};
  if (part < parts) {
#pragma unroll 4
    for (int i = part; i < a.splits; i += parts) {
      const Partial x = of[(int64_t)i * 16];
      const float f = __builtin_amdgcn_exp2f(x.m - use);
      l += x.l * f;
      v += *reinterpret_cast<const f32x4*>(a.part_o + ((slot + i) * 16 + row) * D + d) * __builtin_ldexpf(f, (int)x.e - e_all);
    }
  }
  *reinterpret_cast<f32x4*>(sm_o + 4 * threadIdx.x) = v;
  sm_l[threadIdx.x] = l;
  __syncthreads();
  if (part > 0) return;
  for (int i = 1; i < parts; ++i) {  // in a fixed order
    l += sm_l[threadIdx.x + i * quads];
    v += *reinterpret_cast<const f32x4*>(sm_o + 4 * (threadIdx.x + i * quads));
  }
  const unsigned group = (unsigned)a.group, token = (unsigned)at / group;
  El* to = reinterpret_cast<El*>(a.out) + (sq.row0 + token) * a.o_ts + (int64_t)(h * a.group + (int)((unsigned)at - token * group)) * a.o_hs + d;
  E::store4(to, l == 0.0f ? f32x4{0, 0, 0, 0} : times_two_to(v / l, e_all));  // (a row with a NaN in q has one in l)
}

// Which kernel takes a call, in what pieces.  us on the device, prompt kernel | decode kernel (rows, heads x group, dim; nothing
// held): 300 12x1 64 11.3 | 8.7, 300 2x8 128 13.2 | 12.9, 1200 1x1 64 17.7 | 12.8, 600 2x4 256 35 | 29 -- 300 8x4 128 13.7 | 18.4,
// 600 8x4 128 24 | 37, 2400 12x1 64 58 | 66, 1200 2x4 256 48 | 67: the prompt kernel from half a chip of 64-row pieces on.
// Pieces of 128 rows read and convert codes for twice the rows, but a step takes long with few workgroups on a CU (us, 128 |
// 64 rows): 600 8x4 128 32 | 24, 1200 8x4 128 53 | 38, 2400 12x1 64 80 | 58 -- 2400 8x4 128 87 | 98, 8 x 1000 12x1 64 42 | 47, 2 x 4500
// 4x4 128 288 | 390: 64 while 128 make at most a round of the chip.
// Splits along the tokens (us, one or two workgroups' worth per CU): 300 rows behind 16000 tokens 8x4 128 137 split in six |
// 179 in three, 4 x 40 behind 4000 39 | 48; 1500 behind 500 4x4 128 76 in two | 67 in one, 2400 1x1 64 29 in four, 21 in one: where pieces leave
// half the chip idle, and none of less than 768 tokens.
// The decode kernel's splits fill the chip once with workgroups of eight waves, from 768 tokens on and of at least 256 (us, so |
// twice, of at least 512, the whole in one: one of 2500 tokens 8x4 128 11.8 | 13.1 | 19.1, of 130000 52.9 | 54.3 | -, 8 of 3000
// 17.7 | 20.7 | 23.5, 24 of 2500 8x1 128 30.4 | 32.9 | -; one of 600 in two 12.2, in one 10.6).
// How a call is cut up.
struct AttnPlan {
  int64_t row_tiles, tiles;
  int splits, tile_rows;
  int64_t wg_tiles;  // > 0: row tiles of kv_prompt.hip, of
  int wg_rows;       // so many rows
  size_t ws_bytes;
};
static int plan_attention(const mpq_kv_cache& c, const mpq_kv_batch& b, int type, int q_heads, AttnPlan& p) {
  if (q_heads <= 0 || q_heads % c.heads) return MPQ_ERR_SHAPE;
  const int64_t most = b.max_new < b.rows ? b.max_new : b.rows;
  if (mul_overflows(most, q_heads) || most * (q_heads / c.heads) > 0x7FFFFFFF) return MPQ_ERR_SHAPE;
  p.row_tiles = (most * (q_heads / c.heads) + 15) / 16;
  if (mul_overflows(p.row_tiles, (int64_t)b.seqs * c.heads)) return MPQ_ERR_SHAPE;
  p.tiles = p.row_tiles * b.seqs * c.heads;
  p.splits = 1;
  p.tile_rows = (int)(p.row_tiles > 1 ? 16 : most * (q_heads / c.heads));
  p.wg_tiles = p.wg_rows = 0;
  p.ws_bytes = 0;
  if (p.tiles == 0) return MPQ_OK;
  const int64_t len = b.max_len < (int64_t)b.table_pages * c.page ? b.max_len : (int64_t)b.table_pages * c.page;
  const int64_t pair_rows = most * (q_heads / c.heads), pairs = (int64_t)b.seqs * c.heads;
  auto pieces = [&](int64_t rows) { return (pair_rows + rows - 1) / rows * pairs; };
  const int wide = prompt_rows(type, c.dim);
  const int64_t units = pieces(wide);
  const int64_t cut = (c.dim <= 128 ? 2 : 1) * kNumCU / units, most_cut = len < 768 ? 1 : len / 768;
  const int64_t splits = units > kNumCU / 2 ? 1 : cut < most_cut ? cut : most_cut;
  if (pair_rows >= 128 && pieces(64) * splits >= kNumCU / 2) {
    p.splits = (int)splits;
    p.wg_rows = splits == 1 && units <= 2 * kNumCU && c.dim <= 128 ? 64 : wide;
    p.wg_tiles = (pair_rows + p.wg_rows - 1) / p.wg_rows;
  } else {
    const int64_t want = kNumCU / p.tiles, most_splits = len <= 768 ? 1 : (len + 255) / 256, n = want < most_splits ? want : most_splits;
    p.splits = (int)(n < 1 ? 1 : n);
  }
  if (blocks_z(p.tiles * (p.splits > 16 ? p.splits : 16), 512) > 65535u) return MPQ_ERR_SHAPE;
  p.ws_bytes = p.splits > 1 ? (size_t)p.tiles * p.splits * 16 * (c.dim * sizeof(float) + sizeof(Partial)) : 0;
  return MPQ_OK;
}

template <int T>
static int join(const AttnArgs& a, int64_t tiles, hipStream_t st) {
  kv_attention_join_k<T><<<wide_grid(tiles * a.tile_rows, kBlock), kBlock, 0, st>>>(a);
  return launch_status();
}

template <int T>
static int launch_attention(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const int dh = a.c.dim <= 64 ? 1 : a.c.dim <= 128 ? 2 : 4;
  const bool one = a.c.page >= (dh <= 2 ? 64 : 32);
  // Eight waves where a CU gets one workgroup, four where it gets several (us, 8 | 4 waves, one query each: one sequence of 384
  // tokens 16x1 64 7.1 | 8.0, 8x4 128 8.8 | 9.9, 16 of 500 16x1 64 8.0 | 9.1; 32 of 600 8x4 128 18.5 either way)
  const bool many_waves = dh <= 2 && p.tiles * p.splits <= kNumCU;  // (dim > 128: their shares of the output pass the LDS)
  if (p.wg_tiles == 0) {
    using Kern = void (*)(AttnArgs);
    static const Kern kerns[3][2] = {{kv_attention_k<T, 1, false, 4>, kv_attention_k<T, 1, true, 4>},
                                     {kv_attention_k<T, 2, false, 4>, kv_attention_k<T, 2, true, 4>},
                                     {kv_attention_k<T, 4, false, 4>, kv_attention_k<T, 4, true, 4>}};
    static const Kern wide[2][2] = {{kv_attention_k<T, 1, false, 8>, kv_attention_k<T, 1, true, 8>},
                                    {kv_attention_k<T, 2, false, 8>, kv_attention_k<T, 2, true, 8>}};
    const int threads = many_waves ? 512 : 256;
    const Kern k = many_waves ? wide[dh - 1][one] : kerns[dh >> 1][one];
    k<<<wide_grid(p.tiles * p.splits, threads), threads, 0, st>>>(a);
  }
  const int rc = p.wg_tiles > 0 ? launch_prompt(T, a, p.wg_tiles, p.wg_rows, false, st) : launch_status();
  if (rc != MPQ_OK || p.splits == 1) return rc;
  return join<T>(a, p.tiles, st);
}

int launch_join(int type, const AttnArgs& a, int64_t tiles, hipStream_t st) {
  if (type == MPQ_F32) return join<MPQ_F32>(a, tiles, st);
  return type == MPQ_BF16 ? join<MPQ_BF16>(a, tiles, st) : join<MPQ_F16>(a, tiles, st);
}

int check_rows(const mpq_kv_cache& cache, const mpq_kv_batch& batch, int type, const void* q, int64_t q_token_stride, int64_t q_head_stride,
               int q_heads, const void* out, int64_t out_token_stride, int64_t out_head_stride) {
  if (q_token_stride < 0 || q_head_stride < 0 || out_token_stride < 0 || out_head_stride < 0) return MPQ_ERR_SHAPE;
  if (mul_overflows(batch.rows, q_token_stride) || mul_overflows(batch.rows, out_token_stride) || mul_overflows(q_heads, q_head_stride) ||
      mul_overflows(q_heads, out_head_stride))
    return MPQ_ERR_SHAPE;
  if (batch.rows > 0 && pieces_overlap(batch.rows, out_token_stride, q_heads, out_head_stride, cache.dim)) return MPQ_ERR_SHAPE;
  const uintptr_t el = (uintptr_t)(type_size(type) - 1);
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & el) return MPQ_ERR_ALIGN;
  return MPQ_OK;
}

}  // namespace mpq

using namespace mpq;

extern "C" size_t mpq_kv_attention_workspace_bytes(const mpq_kv_cache* cache, const mpq_kv_batch* batch, int type, int q_heads) {
  AttnPlan p;
  if (check_kv(cache, batch, type) != MPQ_OK || plan_attention(*cache, *batch, type, q_heads, p) != MPQ_OK) return 0;
  return p.ws_bytes;
}

extern "C" int mpq_kv_attention(const mpq_kv_cache* cache, const mpq_kv_batch* batch, int type, const void* q,
                                int64_t q_token_stride, int64_t q_head_stride, int q_heads, float softmax_scale, int causal,
                                int64_t window, void* out, int64_t out_token_stride, int64_t out_head_stride, void* ws,
                                size_t ws_bytes, void* stream) {
  int rc = check_kv(cache, batch, type);
  if (rc != MPQ_OK) return rc;
  AttnPlan p;
  rc = plan_attention(*cache, *batch, type, q_heads, p);
  if (rc != MPQ_OK) return rc;
  if (window < 0 || (window > 0 && !causal) || !(softmax_scale == softmax_scale) || __builtin_isinf(softmax_scale)) return MPQ_ERR_SHAPE;
  rc = check_rows(*cache, *batch, type, q, q_token_stride, q_head_stride, q_heads, out, out_token_stride, out_head_stride);
  if (rc != MPQ_OK) return rc;
  if (p.tiles == 0) return MPQ_OK;
  if (!q || !out) return MPQ_ERR_NULL;
  if (p.ws_bytes > 0 && (!ws || ws_bytes < p.ws_bytes)) return MPQ_ERR_WORKSPACE;
  if (p.ws_bytes > 0 && !aligned16(ws)) return MPQ_ERR_ALIGN;
  AttnArgs a{*cache, *batch, q, q_token_stride, q_head_stride, out, out_token_stride, out_head_stride, q_heads, q_heads / cache->heads,
             causal != 0, cut_window(window), softmax_scale, p.row_tiles, p.splits, p.tile_rows, nullptr, nullptr};
  if (p.splits > 1) {
    a.part_o = reinterpret_cast<float*>(ws);
    a.part = reinterpret_cast<Partial*>(a.part_o + (size_t)p.tiles * p.splits * 16 * cache->dim);
  }
  hipStream_t st = (hipStream_t)stream;
  if (type == MPQ_F32) return launch_attention<MPQ_F32>(a, p, st);
  if (type == MPQ_BF16) return launch_attention<MPQ_BF16>(a, p, st);
  return launch_attention<MPQ_F16>(a, p, st);
}
