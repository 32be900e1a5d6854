// kv_tree.hip -- attention of a tree of drafted tokens over a cache of quantized pages.
//
// The mathematics, the operands' order and the precision are kv_attention.hip's: S' = K q', P, O' = V' P' in registers, one pass over the
// tokens.  A drafted token's rows see the same tokens before the drafted ones, so that a workgroup takes MT tiles of 16 (row, query
// head) pairs: keys and values are read, and their codes made fp16, once for all of them.  The waves deal out the tokens; their shares
// meet in LDS at the end.  Only steps that reach the drafted tokens look at the tree's bits.  Calls with many rows go to
// kv_tree_wide.hip.  Codes' bytes and a workgroup's latency bound it: 5 drafted tokens behind 383, 16 heads of 64 in fp32, 8.4 us from length to
// output; 32 x 5 behind up to 4000, 32 / 8 heads of 128 in bf16, 200 MB in 57 with the one workgroup of eight waves that a CU's share makes.
#include "kv_attn.hpp"

namespace mpq {

constexpr int kTreeBits = 14;  // probabilities are multiplied by 2^14 before they are rounded to fp16

template <int DH, int MT>
struct TreeShape {
  static constexpr int TT = DH * MT <= 2 ? 64 : 32;  // tokens per step
  static constexpr int NW = DH < 4 ? 8 : 4;            // waves (dim > 128: shares of eight pass the LDS)
};

__device__ __forceinline__ v4i stream_codes(const int8_t* p) {
  return __builtin_nontemporal_load((const __attribute__((address_space(1))) v4i*)p);
}

// grid: ((wg tile * seqs + sequence) * heads + head) * splits + split.  DH: dim in units of 64, rounded up.
// ONE: a page holds at least a step's tokens, which then lie on one page.
template <int T, int DH, int MT, bool ONE>
__global__ __launch_bounds__((TreeShape<DH, MT>::NW * 64)) void kv_tree_k(AttnArgs a, TreeMask tree, int64_t wg_tiles) {
  using S = TreeShape<DH, MT>;
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int QT = T == MPQ_F32 ? 2 : 1, TT = S::TT, NS = TT / 16, DP = DH * 64, NW = S::NW, NP = ONE ? 1 : NS;
  __shared__ float sm_m[NW][MT * 16], sm_l[NW][MT * 16];
  __shared__ int sm_e[NW];
  __shared__ __attribute__((aligned(16))) float sm_o[NW / 2][16][DP + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, quarter = lane >> 4;
  const Digits g = digits(a.splits, a.c.heads, a.b.seqs);
  const int split = (int)g.d[0], h = (int)g.d[1];
  const int64_t s = g.d[2], wg_tile = g.d[3];
  if (wg_tile >= wg_tiles) return;
  const Sequence sq = sequence(a.b, a.c.page, (int)s);
  const int64_t len = sq.len < sq.room ? sq.len : sq.room, before = sq.len - sq.n;
  const int64_t room = a.row_tiles * 16, nrows = (int64_t)sq.n * a.group < room ? (int64_t)sq.n * a.group : room;
  const int64_t first_tile = wg_tile * MT;
  if (first_tile * 16 >= nrows) return;
  const int D = a.c.dim;
  const unsigned group = (unsigned)a.group;

  // q: lane (row, quarter) holds channels 64 c + 16 quarter .. + 15 for every c, as the keys come
  f16x8 q[QT][MT][2 * DH];
  float row_scale[MT];
  int64_t tree_row[MT];
  bool real[MT];
#pragma unroll
  for (int n = 0; n < MT; ++n) {
    const int64_t idx = (first_tile + n) * 16 + r;
    real[n] = idx < nrows;
    const unsigned at = real[n] ? (unsigned)idx : 0u, i = at / group;
    tree_row[n] = sq.row0 + i;
    const El* row = reinterpret_cast<const El*>(a.q) + (sq.row0 + i) * a.q_ts + (int64_t)(h * a.group + (int)(at - i * group)) * a.q_hs;
    f32x8 v[2 * DH];
    float m = 0.0f;
#pragma unroll
    for (int c = 0; c < 2 * DH; ++c) {
      const int d = (c >> 1) * 64 + quarter * 16 + (c & 1) * 8;
      v[c] = real[n] && d < D ? E::load8(row + d) : f32x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[c][e]));
    }
    m = fmaxf(m, across(m, 16));
    m = fmaxf(m, across(m, 32));
    const int e2 = kTreeBits - (m > 0.0f ? __builtin_amdgcn_frexp_expf(m) : 0);
#pragma unroll
    for (int c = 0; c < 2 * DH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __builtin_ldexpf(v[c][e], e2);
        const _Float16 top = (_Float16)x;
        q[0][n][c][e] = top;
        if (QT == 2) q[QT - 1][n][c][e] = (_Float16)(x - (float)top);
      }
    // logits in units of log 2
    const float qmax = (float)((1 << (a.c.bits - 1)) - 1);
    row_scale[n] = __builtin_ldexpf(a.scale * kLog2e / qmax, -e2);
  }

  // this workgroup's tokens: whole steps, dealt out to the splits in one piece each and to the waves in turn
  const Span span = {0, len};
  const int64_t all_hi = before < 0 ? 0 : before < len ? before : len;  // what every row sees
  const Steps share = steps_of(span, TT, a.splits, split);
  const int64_t t0 = share.t0, t1 = share.t1;
  const int32_t* table = a.b.table + s * a.b.table_pages;
  const int64_t page_bytes = (int64_t)a.c.page * D;
  const int shift = 31 - __builtin_clz((unsigned)a.c.page);

  // Pages are looked up a step ahead of the codes they hold, codes are requested a step ahead of the products.
  int id[NP];
  auto look_up = [&](int64_t t) {
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int64_t tok = t * TT + u * (TT / NP);
      id[u] = t < t1 && tok < len ? table[tok >> shift] : -1;
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
        kw[u][c] = d < D ? stream_codes(kp[u / (NS / NP)] + (u % (NS / NP) * 16 + r) * D + d) : v4i{0, 0, 0, 0};
      }
  };
  auto request_v = [&]() {
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
      for (int c = 0; c < DH; ++c) {
        const int d = c * 64 + r * 4;
        vw[u][c] = d < D ? stream_codes(vp[u / (NS / NP)] + u % (NS / NP) * 16 * D + (quarter * D + d) * 4) : v4i{0, 0, 0, 0};
      }
  };

  float m_run[MT], l_run[MT];
  int v_exp = -100000;  // O' is in units of 2^(v_exp - kTreeBits)
  f32x4 o[MT][DH][4];
#pragma unroll
  for (int n = 0; n < MT; ++n) {
    m_run[n] = -__builtin_inff();
    l_run[n] = 0.0f;
#pragma unroll
    for (int c = 0; c < DH; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[n][c][k] = f32x4{0, 0, 0, 0};
  }

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
    // S': tokens 16 u + 4 quarter .. + 3 of the step, row r of each tile
    f32x4 sc[MT][NS];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
#pragma unroll
      for (int n = 0; n < MT; ++n) sc[n][u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < DH; ++c) {
        const f16x8 k0 = codes8(kw[u][c].x, kw[u][c].y), k1 = codes8(kw[u][c].z, kw[u][c].w);
#pragma unroll
        for (int x = 0; x < QT; ++x)
#pragma unroll
          for (int n = 0; n < MT; ++n) {
            sc[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[x][n][2 * c], sc[n][u], 0, 0, 0);
            sc[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[x][n][2 * c + 1], sc[n][u], 0, 0, 0);
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
    int ve = v_exp;
#pragma unroll
    for (int u = 0; u < NP; ++u)
      if (mv_now[u] > 0.0f && mv_now[u] < __builtin_inff()) {
        const int e = __builtin_amdgcn_frexp_expf(mv_now[u]);
        ve = e > ve ? e : ve;
      }
    const bool masked = bad || base + TT > all_hi;  // uniform
    f16x4 p[MT][2][NS];
#pragma unroll
    for (int n = 0; n < MT; ++n) {
      // logits, in scalars: see kv_attention.hip
      float x[NS][4];
#pragma unroll
      for (int u = 0; u < NS; ++u) {
        const float f = row_scale[n] * mk_now[u / (NS / NP)];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[u][e] = sc[n][u][e] * f;
      }
      if (masked) {
        // bit 16 u + e: the token 16 u + e behind the lane's first of the step
        const int64_t at = base + quarter * 4, left = len - at;
        uint64_t bits = real[n] ? tree_bits(tree, tree_row[n], at - before) : 0;
        if (left < 64) bits &= left > 0 ? ((uint64_t)1 << left) - 1 : 0;
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool out = !(bits >> (16 * u + e) & 1) | (mk_now[u / (NS / NP)] < 0.0f);
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
      const float m_new = fmaxf(m_run[n], top);
      const float m_use = m_new == -__builtin_inff() ? 0.0f : m_new;
      if (ve != v_exp || __any(m_new > m_run[n])) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[n] - m_use);
        l_run[n] *= alpha;
        const float f = __builtin_ldexpf(alpha, v_exp - ve);
#pragma unroll
        for (int c = 0; c < DH; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[n][c][k] *= f;
        m_run[n] = m_new;
      }
#pragma unroll
      for (int u = 0; u < NS; ++u) {
        // (a maximum of infinity as a factor that leaves a probability of 0 one: rows that see the page become NaN, others do not)
        const float v = mv_now[u / (NS / NP)], f = v > 0.0f ? fminf(__builtin_ldexpf(v, kTreeBits - ve), __FLT_MAX__) : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = __builtin_amdgcn_exp2f(x[u][e] - m_use);
          l_run[n] += w;
          float y = w * f;
          asm("" : "+v"(y));  // its fp32 rounding stays: see kv_attention.hip
          const _Float16 hi16 = (_Float16)y;
          p[n][0][u][e] = hi16;
          p[n][1][u][e] = (_Float16)(y - (float)hi16);
        }
      }
    }
    v_exp = ve;
    // O': channels 64 c + 4 (lane & 15) + k of the value operand
#pragma unroll
    for (int u = 0; u < NS; u += 2) {
#pragma unroll
      for (int c = 0; c < DH; ++c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f16x8 v = codes8(vw[u][c][k], vw[u + 1][c][k]);
#pragma unroll
          for (int term = 0; term < 2; ++term)
#pragma unroll
            for (int n = 0; n < MT; ++n) {
              const f16x8 pp = __builtin_shufflevector(p[n][term][u], p[n][term][u + 1], 0, 1, 2, 3, 4, 5, 6, 7);
              o[n][c][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pp, o[n][c][k], 0, 0, 0);
            }
        }
      }
    }
    if (more) request_v();
  }
  // a row's sum over its four lanes; the waves' shares joined: a lane holds, of row r, channels
  // 64 c + 16 quarter + 4 e + k in o[n][c][k][e]
#pragma unroll
  for (int n = 0; n < MT; ++n) {
    l_run[n] += across(l_run[n], 16);
    l_run[n] += across(l_run[n], 32);
    if (quarter == 0) {
      sm_m[wave][n * 16 + r] = m_run[n];
      sm_l[wave][n * 16 + r] = l_run[n];
    }
  }
  if (lane == 0) sm_e[wave] = v_exp;
  __syncthreads();
  int e_all = sm_e[0];  // shares are added in units of 2^e_all: they are as large as the sum then, whatever the values are
#pragma unroll
  for (int w = 1; w < NW; ++w) e_all = max(e_all, sm_e[w]);
  const float qmax = (float)((1 << (a.c.bits - 1)) - 1);
#pragma unroll
  for (int n = 0; n < MT; ++n) {
    const int64_t tile = first_tile + n;
    if (tile * 16 >= nrows) break;  // uniform
    float m_all = sm_m[0][n * 16 + r];
#pragma unroll
    for (int w = 1; w < NW; ++w) m_all = fmaxf(m_all, sm_m[w][n * 16 + r]);
    const float m_use = m_all == -__builtin_inff() ? 0.0f : m_all;
    const float mine = __builtin_amdgcn_exp2f(m_run[n] - m_use);
    const float f = l_run[n] > 0.0f ? __builtin_ldexpf(mine / qmax, v_exp - e_all - kTreeBits) : 0.0f;
#pragma unroll
    for (int half = 1; half >= 0; --half) {  // the upper half of the waves leaves its share, the lower half adds its own
      if (wave / (NW / 2) == half) {
#pragma unroll
        for (int c = 0; c < DH; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f32x4* to = reinterpret_cast<f32x4*>(&sm_o[wave % (NW / 2)][r][c * 64 + quarter * 16 + 4 * e]);
            const f32x4 v = f32x4{o[n][c][0][e], o[n][c][1][e], o[n][c][2][e], o[n][c][3][e]} * f;
            *to = half ? v : v + *to;
          }
      }
      __syncthreads();
    }
    const int64_t slot = ((s * a.c.heads + h) * a.row_tiles + tile) * a.splits + split;  // of the partial results
    for (int x = threadIdx.x; x < 16 * (D >> 2); x += NW * 64) {
      const int row = x / (D >> 2), d = (x % (D >> 2)) * 4;
      float top = sm_m[0][n * 16 + row];
#pragma unroll
      for (int w = 1; w < NW; ++w) top = fmaxf(top, sm_m[w][n * 16 + row]);
      const float use = top == -__builtin_inff() ? 0.0f : top;
      float l = 0.0f;
      f32x4 v = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < NW; ++w) l += sm_l[w][n * 16 + row] * __builtin_amdgcn_exp2f(sm_m[w][n * 16 + row] - use);
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
    __syncthreads();  // the next tile's shares go to the same place
  }
}

// Joins the splits of a row, a wave per row: its lanes over groups of four channels and, as many as are left, over the splits.  For few splits
// of many rows, where a workgroup per row (kv_attention_join_k) is mostly the launching of workgroups: 9984 rows of two splits of 128
// channels 18.6 us there.
// grid: (((sequence * heads + head) * row_tiles + tile) * tile_rows + row) / 4
template <int T>
__global__ __launch_bounds__(kBlock) void kv_tree_join_k(AttnArgs a) {
  using E = Elem<T>;
  typedef typename E::type El;
  const int lane = threadIdx.x & 63;
  const uint64_t wave = (uint64_t)block_index() * 4 + (uint64_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const Digits g = wave >> 32 == 0 ? split_digits<unsigned>((unsigned)wave, (unsigned)a.tile_rows, (unsigned)a.row_tiles, (unsigned)a.c.heads)
                                   : split_digits<uint64_t>(wave, (uint64_t)a.tile_rows, (uint64_t)a.row_tiles, (uint64_t)a.c.heads);
  const int row = (int)g.d[0], h = (int)g.d[2];
  const int64_t tile = g.d[1], s = g.d[3], slot = ((s * a.c.heads + h) * a.row_tiles + tile) * a.splits;
  if (s >= a.b.seqs) return;
  const Sequence sq = sequence(a.b, a.c.page, (int)s);
  const int64_t at = tile * 16 + row;
  if (at >= joined_rows(a, sq)) return;
  const int D = a.c.dim, quads = D >> 2, parts = kWave / quads, d = lane % quads * 4, part = lane / quads;
  const Partial* of = a.part + slot * 16 + row;  // the row's in the first split; 16 to the next
  float top = -__builtin_inff(), exponent = -__builtin_inff();
  for (int i = lane; i < a.splits; i += kWave) {
    const Partial x = of[(int64_t)i * 16];
    top = fmaxf(top, x.m);
    exponent = fmaxf(exponent, x.e);
  }
  top = wave_max(top);
  const int e_all = (int)wave_max(exponent);
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
  f32x4 sum = v;
  float l_all = l;
  for (int i = 1; i < parts; ++i) {  // in a fixed order
    const int from = (lane + i * quads) & 63;
    l_all += __shfl(l, from, 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += __shfl(v[e], from, 64);
  }
  if (part > 0) return;
  const unsigned group = (unsigned)a.group, token = (unsigned)at / group;
  El* to = reinterpret_cast<El*>(a.out) + (sq.row0 + token) * a.o_ts + (int64_t)(h * a.group + (int)((unsigned)at - token * group)) * a.o_hs + d;
  E::store4(to, l_all == 0.0f ? f32x4{0, 0, 0, 0} : times_two_to(sum / l_all, e_all));  // (a row with a NaN in q has one in l)
}

// Which kernel takes a call, in what pieces: up to 32 rows (row, query head pairs of a key head) the one here, with one or two tiles and splits
// that fill the chip once; more in the wide kernel, in pieces of 64 rows of which three workgroups share a CU, of 128 from 129 rows on; few
// rows over short sequences here, where a workgroup's latency counts.  us on the device, bf16, pages of 64 (sequences x drafted
// tokens behind held, key heads x group, dim; one tile | two tiles | pieces of 64 | of 128, each with its best number of splits):
// 1 x 3 behind 60000 8x4 128 fp16 33 | 34 | 42 | 56, 32 x 5 behind 4000 8x4 128 74 | 56 | 69 | 101, 1 x 5 behind 32000 29 | 27 | 29 | 39, 8 x 7 behind 8000 44 |
// 39 | 43 | 59, 32 x 30 behind 1000 12x1 64 29 | 26 | 28 | 39 -- 4 x 16 behind 8000 8x4 128 41 | 38 | 31 | 39, 24 x 13 behind 8000 173 | 145 | 95 | 142, the
// same behind 4000 in fp32 102 | 92 | 71 | -, 4 x 30 behind 8000 61 | 59 | 46 | 46, 16 x 60 behind 2000 8x8 128 249 | 174 | 94 | 103, 1 x 61 behind 65500 8x4 128
// fp16 235 | 185 | 140 | 121, 2 x 10 behind 16000 2x7 256 45 | - | - | 33 -- 1 x 60 behind 400 12x1 64 7.7 | 10.6 | 14 | 18, 2 x 100 behind 300 8x4 128 18.8 |
// 15.0 | 18.9 | 26.  (16 x 60 would be better off with pieces of 64.  Four tiles here, which need 480 registers: 24 x 13 behind 8000 196.)  Splits: 4 x 16
// behind 8000 in pieces of 64, 8 | 16 | 32: 34 | 31 | 38; 24 x 13 behind 8000, 2 | 4 | 8: 123 | 95 | 97.
struct TreePlan {
  int64_t row_tiles, tiles, wg_tiles;
  int mt, splits, tile_rows;
  int wide_rows;  // > 0: kv_tree_wide.hip, workgroups of so many rows
  size_t ws_bytes;
};
static int plan_tree(const mpq_kv_cache& c, const mpq_kv_batch& b, int type, int q_heads, TreePlan& p) {
  if (q_heads <= 0 || q_heads % c.heads) return MPQ_ERR_SHAPE;
  const int64_t most = b.max_new < b.rows ? b.max_new : b.rows;
  if (mul_overflows(most, q_heads) || most * (q_heads / c.heads) > 0x7FFFFFFF) return MPQ_ERR_SHAPE;
  const int64_t pair_rows = most * (q_heads / c.heads), pairs = (int64_t)b.seqs * c.heads;
  p.row_tiles = (pair_rows + 15) / 16;
  if (mul_overflows(p.row_tiles, pairs)) return MPQ_ERR_SHAPE;
  p.tiles = p.row_tiles * pairs;
  p.splits = 1;
  p.tile_rows = (int)(p.row_tiles > 1 ? 16 : pair_rows);
  p.wide_rows = 0;
  p.ws_bytes = 0;
  if (p.tiles == 0) return MPQ_OK;
  const int64_t room = (int64_t)b.table_pages * c.page, len = b.max_len < room ? b.max_len : room;
  // a workgroup's row tiles here; few, short sequences' rows spread over the chip
  const bool narrow = c.dim <= 128;
  p.mt = p.row_tiles == 1 || !narrow || (len <= 768 && pair_rows > 32 && p.tiles <= kNumCU) ? 1 : 2;
  p.wg_tiles = (p.row_tiles + p.mt - 1) / p.mt;
  const int64_t units = p.wg_tiles * pairs;
  int64_t splits = kNumCU / units, most_splits = len <= 768 ? 1 : (len + 255) / 256;
  if (pair_rows > 32 && !(len <= 768 && units <= kNumCU)) {
    const int wide = prompt_rows(type, c.dim);
    p.wide_rows = narrow && pair_rows <= 128 ? 64 : wide;
    p.wg_tiles = (pair_rows + p.wide_rows - 1) / p.wide_rows;
    splits = (!narrow ? 1 : p.wide_rows == 64 ? 3 : 2) * kNumCU / (p.wg_tiles * pairs);
    most_splits = len < 1000 ? 1 : len / 500;
  }
  splits = splits < most_splits ? splits : most_splits;
  p.splits = (int)(splits < 1 ? 1 : splits);
  if (blocks_z(p.tiles * (p.splits > 16 ? p.splits : 16), 512) > 65535u) return MPQ_ERR_SHAPE;
  p.ws_bytes = p.splits > 1 ? (size_t)p.tiles * p.splits * 16 * (c.dim * sizeof(float) + sizeof(Partial)) : 0;
  return MPQ_OK;
}

template <int T, int DH, int MT>
static int go(const AttnArgs& a, const TreeMask& tree, int64_t wg_tiles, hipStream_t st) {
  using S = TreeShape<DH, MT>;
  const dim3 grid = wide_grid(wg_tiles * a.b.seqs * a.c.heads * a.splits, S::NW * 64);
  if (a.c.page >= S::TT) kv_tree_k<T, DH, MT, true><<<grid, S::NW * 64, 0, st>>>(a, tree, wg_tiles);
  else kv_tree_k<T, DH, MT, false><<<grid, S::NW * 64, 0, st>>>(a, tree, wg_tiles);
  return launch_status();
}
template <int T, int DH>
static int go_tiles(const AttnArgs& a, const TreeMask& tree, const TreePlan& p, hipStream_t st) {
  if constexpr (DH < 4) {
    if (p.mt == 2) return go<T, DH, 2>(a, tree, p.wg_tiles, st);
  }
  return go<T, DH, 1>(a, tree, p.wg_tiles, st);
}
template <int T>
static int launch_tree(const AttnArgs& a, const TreeMask& tree, const TreePlan& p, hipStream_t st) {
  int rc;
  if (p.wide_rows > 0) rc = launch_tree_wide(T, a, tree, p.wg_tiles, p.wide_rows, st);
  else if (a.c.dim <= 64) rc = go_tiles<T, 1>(a, tree, p, st);
  else rc = a.c.dim <= 128 ? go_tiles<T, 2>(a, tree, p, st) : go_tiles<T, 4>(a, tree, p, st);
  if (rc != MPQ_OK || p.splits == 1) return rc;
  if (p.splits > 16) return launch_join(T, a, p.tiles, st);
  kv_tree_join_k<T><<<wide_grid((p.tiles * p.tile_rows + 3) / 4, kBlock), kBlock, 0, st>>>(a);
  return launch_status();
}

}  // namespace mpq

using namespace mpq;

extern "C" size_t mpq_kv_attention_tree_workspace_bytes(const mpq_kv_cache* cache, const mpq_kv_batch* batch, int type, int q_heads) {
  TreePlan p;
  if (check_kv(cache, batch, type) != MPQ_OK || plan_tree(*cache, *batch, type, q_heads, p) != MPQ_OK) return 0;
  return p.ws_bytes;
}

extern "C" int mpq_kv_attention_tree(const mpq_kv_cache* cache, const mpq_kv_batch* batch, int type, const void* q, int64_t q_token_stride,
                                     int64_t q_head_stride, int q_heads, float softmax_scale, const int64_t* tree, int tree_words,
                                     void* out, int64_t out_token_stride, int64_t out_head_stride, void* ws, size_t ws_bytes,
                                     void* stream) {
  int rc = check_kv(cache, batch, type);
  if (rc != MPQ_OK) return rc;
  TreePlan p;
  rc = plan_tree(*cache, *batch, type, q_heads, p);
  if (rc != MPQ_OK) return rc;
  if (!(softmax_scale == softmax_scale) || __builtin_isinf(softmax_scale)) return MPQ_ERR_SHAPE;
  if (tree_words < 1 || mul_overflows(batch->rows, tree_words)) return MPQ_ERR_SHAPE;
  rc = check_rows(*cache, *batch, type, q, q_token_stride, q_head_stride, q_heads, out, out_token_stride, out_head_stride);
  if (rc != MPQ_OK) return rc;
  if (reinterpret_cast<uintptr_t>(tree) & 7u) return MPQ_ERR_ALIGN;
  if (p.tiles == 0) return MPQ_OK;
  if (!q || !out || !tree) return MPQ_ERR_NULL;
  if (p.ws_bytes > 0 && (!ws || ws_bytes < p.ws_bytes)) return MPQ_ERR_WORKSPACE;
  if (p.ws_bytes > 0 && !aligned16(ws)) return MPQ_ERR_ALIGN;
  AttnArgs a{*cache, *batch, q, q_token_stride, q_head_stride, out, out_token_stride, out_head_stride, q_heads, q_heads / cache->heads, 0,
             0, softmax_scale, p.row_tiles, p.splits, p.tile_rows, nullptr, nullptr};
  const TreeMask mask{reinterpret_cast<const uint64_t*>(tree), tree_words};
  if (p.splits > 1) {
    a.part_o = reinterpret_cast<float*>(ws);
    a.part = reinterpret_cast<Partial*>(a.part_o + (size_t)p.tiles * p.splits * 16 * cache->dim);
  }
  hipStream_t st = (hipStream_t)stream;
  if (type == MPQ_F32) return launch_tree<MPQ_F32>(a, mask, p, st);
  if (type == MPQ_BF16) return launch_tree<MPQ_BF16>(a, mask, p, st);
  return launch_tree<MPQ_F16>(a, mask, p, st);
}
