// kv_cache.hip -- keys and values into a cache of quantized pages, and back out of it.
//
// A workgroup owns one page of one sequence and head, for keys or for values, so that nobody else writes its bytes.  A thread
// holds eight channels of four tokens in registers: a workgroup has as many threads as the rows may touch such pieces of a page,
// and rows are read once.  It takes their maximum, forms the page's new maximum, and writes codes.  Codes already there are
// read and written again only where the maximum grew.
// Value codes lie four tokens of a channel to a dword (the order the attention's product wants its operand in): a thread's
// piece is 32 bytes, which it merges into what is there.
// Bound by the bytes of the rows and codes for prompts: 7 ragged prompts of up to 2600 rows of 2 x 12 x 64 fp32 in 24.8 us
// (84 MB read, 21 written: 4.2 TB/s; rows read twice, by 256 threads a page, 32 us), back out of the cache in 21.3 (4.9 TB/s).
// For single tokens bound by three dependent loads (length, table, maximum) and the launch: one of each of 128 sequences 6 us.
#include "kv.hpp"

namespace mpq {

typedef int v4i __attribute__((ext_vector_type(4)));

int check_kv(const mpq_kv_cache* c, const mpq_kv_batch* b, int type) {
  if (!c || !b) return MPQ_ERR_NULL;
  if (!known_type(type)) return MPQ_ERR_SHAPE;
  if (c->pages <= 0 || c->heads <= 0 || c->dim <= 0 || c->dim > 256 || c->dim % 16) return MPQ_ERR_SHAPE;
  if (c->heads > 0x3FFFFFFF) return MPQ_ERR_SHAPE;  // (a grid counts keys' and values' heads)
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return MPQ_ERR_SHAPE;
  if (mul_overflows(c->pages, (int64_t)c->heads) || mul_overflows(c->pages * c->heads, (int64_t)c->page * c->dim)) return MPQ_ERR_SHAPE;
  if (c->bits < 2 || c->bits > 8) return MPQ_ERR_BITS;
  if (b->rows < 0 || b->seqs < 0 || b->table_pages <= 0 || b->max_new < 0 || b->max_len < 0) return MPQ_ERR_SHAPE;
  if (b->rows > 0x7FFFFFFF || b->max_new > 0x7FFFFFFF || b->max_len > 0x7FFFFFFF) return MPQ_ERR_SHAPE;
  if (!c->k_codes || !c->v_codes || !c->k_absmax || !c->v_absmax) return MPQ_ERR_NULL;
  if (b->seqs > 0 && (!b->starts || !b->kv_len || !b->table)) return MPQ_ERR_NULL;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return MPQ_ERR_ALIGN;
  for (const void* p : {(const void*)c->k_absmax, (const void*)c->v_absmax, (const void*)b->starts, (const void*)b->kv_len,
                        (const void*)b->table})
    if (reinterpret_cast<uintptr_t>(p) & 3u) return MPQ_ERR_ALIGN;
  return MPQ_OK;
}

// a page of a sequence that a call's rows touch
struct PageRows {
  int64_t at;    // its place in the sequence's row of the table
  int lo, hi;    // places lo .. hi - 1 on it are the call's rows
  int64_t row;   // row of place lo
};
// The j-th page of a sequence that its rows lie on; false: there is none.
__device__ __forceinline__ bool page_rows(const Sequence& q, int page, int64_t j, PageRows& p) {
  const int64_t before = q.len - q.n, first = before < 0 ? 0 : before;
  const int64_t at = (first >> __builtin_ctz(page)) + j, end = q.len < q.room ? q.len : q.room;
  if (at * page >= end) return false;
  const int64_t lo = first > at * page ? first : at * page, hi = end < (at + 1) * page ? end : (at + 1) * page;
  if (lo >= hi) return false;
  p.at = at;
  p.lo = (int)(lo - at * page);
  p.hi = (int)(hi - at * page);
  p.row = q.row0 + (lo - before);
  return true;
}

// where a workgroup works
struct Place {
  int64_t j, s;  // page of the sequence, sequence
  int h;         // head
};
template <typename I>
__device__ __forceinline__ Place split_index(I g, I heads, I pages_per_seq) {
  Place w;
  w.h = (int)(g % heads);
  g /= heads;
  w.j = (int64_t)(g % pages_per_seq);
  w.s = (int64_t)(g / pages_per_seq);
  return w;
}
// (a 64-bit division is 150 scalar instructions, and the waves of a SIMD share its scalar unit: reading back 128 x
// 64 rows of 8 heads 18.8 -> 16.9 us)
__device__ __forceinline__ Place place_of(int heads, int64_t pages_per_seq) {
  if (gridDim.z == 1) return split_index<unsigned>(blockIdx.x, (unsigned)heads, (unsigned)pages_per_seq);
  return split_index<uint64_t>((uint64_t)block_index(), (uint64_t)heads, (uint64_t)pages_per_seq);
}

__device__ __forceinline__ float byte_of(int w, int e) { return (float)(int8_t)((unsigned)w >> (8 * e)); }

constexpr int kMaxKvThreads = 1024;  // a page of 128 tokens of 256 channels

// grid: seqs * pages_per_seq * (2 * heads), keys' heads first
template <int T>
__global__ __launch_bounds__(kMaxKvThreads) void kv_append_k(mpq_kv_cache c, mpq_kv_batch b, int64_t pages_per_seq,
                                                             const void* __restrict__ kv, int64_t k_ts, int64_t k_hs,
                                                             const void* __restrict__ vv, int64_t v_ts, int64_t v_hs) {
  using E = Elem<T>;
  typedef typename E::type El;
  __shared__ float sm[kMaxKvThreads / kWave];
  Place w = place_of(2 * c.heads, pages_per_seq);
  if (w.s >= b.seqs) return;
  const bool values = w.h >= c.heads;
  if (values) w.h -= c.heads;
  PageRows p;
  if (!page_rows(sequence(b, c.page, (int)w.s), c.page, w.j, p)) return;
  const int64_t id = b.table[w.s * b.table_pages + p.at];
  const int D = c.dim, eights = D >> 3;
  const int64_t ts = values ? v_ts : k_ts;
  const El* x = reinterpret_cast<const El*>(values ? vv : kv) + p.row * ts + w.h * (values ? v_hs : k_hs);  // place lo
  // the thread's four tokens and eight channels
  const int grp = (p.lo >> 2) + (int)threadIdx.x / eights, at = ((int)threadIdx.x % eights) * 8;
  const bool mine = 4 * grp < p.hi;
  f32x8 f[4];
  float m = 0.0f;
  if (mine) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {  // (a place that is not the call's: a row that is, which changes no maximum)
      const int place = 4 * grp + t;
      f[t] = E::load8(x + ((place < p.lo ? p.lo : place < p.hi ? place : p.hi - 1) - p.lo) * ts + at);
    }
  }
  if (id < 0 || id >= c.pages) return;
  float* absmax = (values ? c.v_absmax : c.k_absmax) + id * c.heads + w.h;
  int8_t* codes = (values ? c.v_codes : c.k_codes) + (id * c.heads + w.h) * ((int64_t)c.page * D);
  const float was = p.lo > 0 ? *absmax : 0.0f;
  // values: what is there already, also bytes behind the last token, which stay as they are (requested with the maximum: for a
  // single token each memory access that waits for another counts)
  v4i* to = reinterpret_cast<v4i*>(codes + (grp * D + at) * 4);
  v4i v[2] = {v4i{0, 0, 0, 0}, v4i{0, 0, 0, 0}};
  if (values && mine && (4 * grp < p.lo || 4 * grp + 4 > p.hi)) {
    v[0] = to[0];
    v[1] = to[1];
  }
  if (mine) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(f[t][e]));
  }
  m = wave_max(m);
  if (blockDim.x > kWave) {
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
    __syncthreads();
    for (int i = 0; i < (int)(blockDim.x >> 6); ++i) m = fmaxf(m, sm[i]);
  }
  m = fmaxf(m, was);
  float scale, inv, old_scale, old_inv;
  step_constants(m, c.bits, scale, inv);
  step_constants(was, c.bits, old_scale, old_inv);
  const float qmax = (float)((1 << (c.bits - 1)) - 1);
  auto requant = [&](int v, int e) { return (unsigned)(int)code_f(byte_of(v, e) * old_scale, inv, qmax) & 0xFFu; };
  const bool again = p.lo > 0 && m > was;
  if (again) {  // whole keys, or whole groups of values, that were there before
    const int n = (values ? p.lo & ~3 : p.lo) * (D >> 4);
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      v4i v = *reinterpret_cast<const v4i*>(codes + i * 16);
#pragma unroll
      for (int d = 0; d < 4; ++d) v[d] = (int)(requant(v[d], 0) | requant(v[d], 1) << 8 | requant(v[d], 2) << 16 | requant(v[d], 3) << 24);
      *reinterpret_cast<v4i*>(codes + i * 16) = v;
    }
  }
  if (mine && !values) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int place = 4 * grp + t;
      if (place >= p.lo && place < p.hi)
        *reinterpret_cast<v2i*>(codes + place * D + at) = v2i{(int)pack_codes(f[t][0], f[t][1], f[t][2], f[t][3], inv, qmax),
                                                              (int)pack_codes(f[t][4], f[t][5], f[t][6], f[t][7], inv, qmax)};
    }
  } else if (mine) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int before = v[e >> 2][e & 3];
      unsigned d = 0;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int place = 4 * grp + t;
        const unsigned held = again && place < p.lo ? requant(before, t) : (unsigned)before >> (8 * t) & 0xFFu;
        const unsigned fresh = (unsigned)(int)code_f(f[t][e], inv, qmax) & 0xFFu;
        d |= (place >= p.lo && place < p.hi ? fresh : held) << (8 * t);
      }
      v[e >> 2][e & 3] = (int)d;
    }
    to[0] = v[0];
    to[1] = v[1];
  }
  if (threadIdx.x == 0) *absmax = m;  // (everyone has read it: the barrier, or the one wave)
}

// A workgroup takes a page's keys and its values: twice the loads in flight behind the same look-ups, and half the waves
// (128 sequences of up to 64 rows of 8 x 128 channels 16.9 -> 10.6 us).  grid: seqs * pages_per_seq * heads.  Rows of absent
// tokens become 0.
template <int T>
__global__ __launch_bounds__(kMaxKvThreads) void kv_gather_k(mpq_kv_cache c, mpq_kv_batch b, int64_t pages_per_seq,
                                                             void* __restrict__ k_out, void* __restrict__ v_out) {
  using E = Elem<T>;
  typedef typename E::type El;
  const Place w = place_of(c.heads, pages_per_seq);
  if (w.s >= b.seqs) return;
  const int D = c.dim, eights = D >> 3;
  const int64_t ts = (int64_t)c.heads * D;
  El* k_to = reinterpret_cast<El*>(k_out) + w.h * D;
  El* v_to = reinterpret_cast<El*>(v_out) + w.h * D;
  const Sequence q = sequence(b, c.page, (int)w.s);
  PageRows p;
  if (page_rows(q, c.page, w.j, p)) {
    const int64_t id = b.table[w.s * b.table_pages + p.at];
    const bool there = id >= 0 && id < c.pages;
    const int64_t page = (there ? id : 0) * c.heads + w.h;
    const float k_max = c.k_absmax[page], v_max = c.v_absmax[page];
    const int64_t base = page * ((int64_t)c.page * D);
    const int grp = (p.lo >> 2) + (int)threadIdx.x / eights, at = ((int)threadIdx.x % eights) * 8;
    if (4 * grp < p.hi) {
      v2i kw[4];  // (a page holds whole groups)
      v4i vw[2];
      if (k_out) {
#pragma unroll
        for (int t = 0; t < 4; ++t) kw[t] = *reinterpret_cast<const v2i*>(c.k_codes + base + (4 * grp + t) * D + at);
      }
      if (v_out) {
#pragma unroll
        for (int e = 0; e < 2; ++e) vw[e] = *reinterpret_cast<const v4i*>(c.v_codes + base + (grp * D + at + 4 * e) * 4);
      }
      float k_step, v_step, inv;
      step_constants(k_max, c.bits, k_step, inv);
      step_constants(v_max, c.bits, v_step, inv);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int place = 4 * grp + t;
        if (place < p.lo || place >= p.hi) continue;
        const int64_t row = (p.row + place - p.lo) * ts + at;
        f32x8 f;
        if (k_out) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = there ? byte_of(kw[t][e >> 2], e & 3) * k_step : 0.0f;
          E::store8(k_to + row, f);
        }
        if (v_out) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = there ? byte_of(vw[e >> 2][e & 3], t) * v_step : 0.0f;
          E::store8(v_to + row, f);
        }
      }
    }
  }
  // rows without a place: in front of the sequence's first token, behind the table's last
  const int64_t before = q.len - q.n;
  if (w.j == 0 && (before < 0 || q.len > q.room)) {
    for (int64_t i = 0; i < q.n; ++i)
      if (before + i < 0 || before + i >= q.room)
        for (int d = threadIdx.x; d < D; d += blockDim.x) {
          if (k_out) k_to[(q.row0 + i) * ts + d] = (El)0.0f;
          if (v_out) v_to[(q.row0 + i) * ts + d] = (El)0.0f;
        }
  }
}

// Workgroups of a call: pages that max_new rows of a sequence may touch, sequences, per_page of a page; threads: one for
// each four tokens and eight channels that the rows may touch on a page.
static int kv_grid(const mpq_kv_cache& c, const mpq_kv_batch& b, int64_t per_page, int& threads, int64_t& pages_per_seq, dim3& grid) {
  const int64_t most = b.max_new < b.rows ? b.max_new : b.rows;
  const int64_t groups = (most + 2) / 4 + 1;
  threads = (int)(((groups < c.page / 4 ? groups : c.page / 4) * (c.dim / 8) + kWave - 1) / kWave * kWave);
  pages_per_seq = (most + c.page - 2) / c.page + 1;
  if (pages_per_seq > b.table_pages) pages_per_seq = b.table_pages;
  int64_t want;
  if (__builtin_mul_overflow(pages_per_seq * b.seqs, per_page, &want) || want > ((int64_t)1 << 40)) return MPQ_ERR_SHAPE;
  if (blocks_z(want, threads) > 65535u) return MPQ_ERR_SHAPE;
  grid = wide_grid(want, threads);
  return MPQ_OK;
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_kv_append(const mpq_kv_cache* cache, const mpq_kv_batch* batch, int type, const void* k, int64_t k_token_stride,
                             int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride, void* stream) {
  int rc = check_kv(cache, batch, type);
  if (rc != MPQ_OK) return rc;
  const uintptr_t el = (uintptr_t)(type_size(type) - 1);
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & el) return MPQ_ERR_ALIGN;
  if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0) return MPQ_ERR_SHAPE;
  if (mul_overflows(batch->rows, k_token_stride) || mul_overflows(batch->rows, v_token_stride) ||
      mul_overflows(cache->heads, k_head_stride) || mul_overflows(cache->heads, v_head_stride))
    return MPQ_ERR_SHAPE;
  if (batch->rows == 0 || batch->seqs == 0 || batch->max_new == 0) return MPQ_OK;
  if (!k || !v) return MPQ_ERR_NULL;
  int64_t pages;
  int threads;
  dim3 grid;
  rc = kv_grid(*cache, *batch, (int64_t)2 * cache->heads, threads, pages, grid);
  if (rc != MPQ_OK) return rc;
  const auto kernel = type == MPQ_F32 ? kv_append_k<MPQ_F32> : type == MPQ_BF16 ? kv_append_k<MPQ_BF16> : kv_append_k<MPQ_F16>;
  kernel<<<grid, threads, 0, (hipStream_t)stream>>>(*cache, *batch, pages, k, k_token_stride, k_head_stride, v, v_token_stride,
                                                    v_head_stride);
  return launch_status();
}

extern "C" int mpq_kv_gather(const mpq_kv_cache* cache, const mpq_kv_batch* batch, int type, void* k_out, void* v_out, void* stream) {
  int rc = check_kv(cache, batch, type);
  if (rc != MPQ_OK) return rc;
  const uintptr_t el = (uintptr_t)(type_size(type) - 1);
  if ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & el) return MPQ_ERR_ALIGN;
  if (mul_overflows(batch->rows, (int64_t)cache->heads * cache->dim)) return MPQ_ERR_SHAPE;
  if (batch->rows == 0 || batch->seqs == 0 || batch->max_new == 0) return MPQ_OK;
  if (!k_out && !v_out) return MPQ_ERR_NULL;
  int64_t pages;
  int threads;
  dim3 grid;
  rc = kv_grid(*cache, *batch, cache->heads, threads, pages, grid);
  if (rc != MPQ_OK) return rc;
  const auto kernel = type == MPQ_F32 ? kv_gather_k<MPQ_F32> : type == MPQ_BF16 ? kv_gather_k<MPQ_BF16> : kv_gather_k<MPQ_F16>;
  kernel<<<grid, threads, 0, (hipStream_t)stream>>>(*cache, *batch, pages, k_out, v_out);
  return launch_status();
}
