// kv_cache.hip -- keys and values into a cache of quantized pages, and back out of it.
//
// A workgroup owns one page of one sequence and head, for keys or for values, so that nobody else writes its bytes: it takes
// the maximum of the new rows (a first read), forms the page's new maximum, and writes codes (a second read of the rows,
// out of the caches).  Codes already there are read and written again only where the maximum grew.
// Value codes lie four tokens of a channel to a dword (the order the attention's product wants its operand in); a
// lane owns 16 bytes, four channels of four tokens, and merges what is new into what is there.
// Bound by the bytes of the rows and codes for prompts; for single tokens by three dependent loads (length, table and
// maximum) and the launch.
#include "kv.hpp"

namespace mpq {

typedef int v4i __attribute__((ext_vector_type(4)));

int check_kv(const mpq_kv_cache* c, const mpq_kv_batch* b, int type) {
  if (!c || !b) return MPQ_ERR_NULL;
  if (!known_type(type)) return MPQ_ERR_SHAPE;
  if (c->pages <= 0 || c->heads <= 0 || c->dim <= 0 || c->dim > 256 || c->dim % 16) return MPQ_ERR_SHAPE;
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
  int64_t id;    // the page
  int lo, hi;    // places lo .. hi - 1 on it are the call's rows
  int64_t row;   // row of place lo
};
// The j-th page of sequence s that its rows lie on; false: there is none.  id < 0 or >= pages: a page that does not exist.
__device__ __forceinline__ bool page_rows(const mpq_kv_batch& b, int page, int s, int64_t j, PageRows& p) {
  const Sequence q = sequence(b, page, s);
  const int64_t before = q.len - q.n, first = before < 0 ? 0 : before;
  const int64_t at = first / page + j, end = q.len < q.room ? q.len : q.room;
  if (at * page >= end) return false;
  const int64_t lo = first > at * page ? first : at * page, hi = end < (at + 1) * page ? end : (at + 1) * page;
  if (lo >= hi) return false;
  p.id = b.table[(int64_t)s * b.table_pages + at];
  p.lo = (int)(lo - at * page);
  p.hi = (int)(hi - at * page);
  p.row = q.row0 + (lo - before);
  return true;
}

__device__ __forceinline__ float byte_of(int w, int e) { return (float)(int8_t)((unsigned)w >> (8 * e)); }

// NT threads: a wave where a call brings a token or two, else 256.  grid: seqs * pages_per_seq * heads * 2, values last.
template <int T, int NT>
__global__ __launch_bounds__(NT) void kv_append_k(mpq_kv_cache c, mpq_kv_batch b, int64_t pages_per_seq, const void* __restrict__ kv,
                                                  int64_t k_ts, int64_t k_hs, const void* __restrict__ vv, int64_t v_ts, int64_t v_hs) {
  using E = Elem<T>;
  typedef typename E::type El;
  __shared__ float sm[NT / kWave];
  int64_t g = block_index();
  const bool values = g & 1;
  g >>= 1;
  const int h = (int)(g % c.heads);
  g /= c.heads;
  const int64_t j = g % pages_per_seq;
  const int64_t s = g / pages_per_seq;
  if (s >= b.seqs) return;
  PageRows p;
  if (!page_rows(b, c.page, (int)s, j, p) || p.id < 0 || p.id >= c.pages) return;
  const int D = c.dim;
  const int64_t ts = values ? v_ts : k_ts;
  const El* x = reinterpret_cast<const El*>(values ? vv : kv) + p.row * ts + h * (values ? v_hs : k_hs);  // place lo
  float* absmax = (values ? c.v_absmax : c.k_absmax) + p.id * c.heads + h;
  int8_t* codes = (values ? c.v_codes : c.k_codes) + (p.id * c.heads + h) * ((int64_t)c.page * D);
  const float was = p.lo > 0 ? *absmax : 0.0f;

  float m = 0.0f;
  const int per_row = D >> 3, total = (p.hi - p.lo) * per_row;
  for (int i = threadIdx.x; i < total; i += NT) {
    const int t = i / per_row;
    const f32x8 w = E::load8(x + t * ts + (i - t * per_row) * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(w[e]));
  }
  m = wave_max(m);
  if (NT > kWave) {
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
    __syncthreads();
    for (int i = 0; i < NT / kWave; ++i) m = fmaxf(m, sm[i]);
  }
  m = fmaxf(m, was);
  float scale, inv, old_scale, old_inv;
  step_constants(m, c.bits, scale, inv);
  step_constants(was, c.bits, old_scale, old_inv);
  const float qmax = (float)((1 << (c.bits - 1)) - 1);
  const bool again = p.lo > 0 && m > was;
  auto requant = [&](int w, int e) { return (unsigned)(int)code_f(byte_of(w, e) * old_scale, inv, qmax) & 0xFFu; };

  if (!values) {
    if (again) {
      const int n = p.lo * (D >> 4);
      for (int i = threadIdx.x; i < n; i += NT) {
        v4i w = *reinterpret_cast<const v4i*>(codes + i * 16);
#pragma unroll
        for (int d = 0; d < 4; ++d) w[d] = (int)(requant(w[d], 0) | requant(w[d], 1) << 8 | requant(w[d], 2) << 16 | requant(w[d], 3) << 24);
        *reinterpret_cast<v4i*>(codes + i * 16) = w;
      }
    }
    for (int i = threadIdx.x; i < total; i += NT) {
      const int t = i / per_row, at = (i - t * per_row) * 8;
      const f32x8 w = E::load8(x + t * ts + at);
      *reinterpret_cast<v2i*>(codes + (p.lo + t) * D + at) =
          v2i{(int)pack_codes(w[0], w[1], w[2], w[3], inv, qmax), (int)pack_codes(w[4], w[5], w[6], w[7], inv, qmax)};
    }
  } else {
    const int quads = D >> 2, g0 = again ? 0 : p.lo >> 2, g1 = (p.hi + 3) >> 2;
    for (int i = threadIdx.x; i < (g1 - g0) * quads; i += NT) {
      const int grp = g0 + i / quads, at = (i % quads) * 4;
      v4i* to = reinterpret_cast<v4i*>(codes + (grp * D + at) * 4);
      // what is there already: also bytes behind the last token, which stay as they are
      v4i w = 4 * grp < p.lo || 4 * grp + 4 > p.hi ? *to : v4i{0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int place = 4 * grp + t;
        const unsigned keep = ~(0xFFu << (8 * t));
        if (place < p.lo) {
          if (again)
            for (int d = 0; d < 4; ++d) w[d] = (int)(((unsigned)w[d] & keep) | requant(w[d], t) << (8 * t));
        } else if (place < p.hi) {
          const f32x4 f = E::load4(x + (place - p.lo) * ts + at);
          for (int d = 0; d < 4; ++d) w[d] = (int)(((unsigned)w[d] & keep) | ((unsigned)(int)code_f(f[d], inv, qmax) & 0xFFu) << (8 * t));
        }
      }
      *to = w;
    }
  }
  if (threadIdx.x == 0) *absmax = m;  // (everyone has read it: the barrier, or the one wave)
}

// grid as kv_append_k.  Rows of absent tokens become 0.
template <int T>
__global__ __launch_bounds__(kBlock) void kv_gather_k(mpq_kv_cache c, mpq_kv_batch b, int64_t pages_per_seq, void* __restrict__ kv,
                                                      void* __restrict__ vv) {
  using E = Elem<T>;
  typedef typename E::type El;
  int64_t g = block_index();
  const bool values = g & 1;
  g >>= 1;
  const int h = (int)(g % c.heads);
  g /= c.heads;
  const int64_t j = g % pages_per_seq;
  const int64_t s = g / pages_per_seq;
  El* out = reinterpret_cast<El*>(values ? vv : kv);
  if (s >= b.seqs || !out) return;
  const int D = c.dim;
  const int64_t ts = (int64_t)c.heads * D;
  out += h * D;
  if (j == 0) {  // rows without a place: in front of the sequence's first token, behind the table's last
    const Sequence q = sequence(b, c.page, (int)s);
    const int64_t before = q.len - q.n;
    for (int64_t i = 0; i < q.n; ++i) {
      if (before + i >= 0 && before + i < q.room) {
        if (before >= 0 && q.len <= q.room) break;  // all of them have one
        continue;
      }
      for (int d = threadIdx.x; d < D; d += kBlock) out[(q.row0 + i) * ts + d] = (El)0.0f;
    }
  }
  PageRows p;
  if (!page_rows(b, c.page, (int)s, j, p)) return;
  const bool there = p.id >= 0 && p.id < c.pages;
  const int64_t at = ((there ? p.id : 0) * c.heads + h);
  float scale, inv;
  step_constants((values ? c.v_absmax : c.k_absmax)[at], c.bits, scale, inv);
  const int8_t* codes = (values ? c.v_codes : c.k_codes) + at * ((int64_t)c.page * D);
  out += p.row * ts;
  if (!values) {
    const int per_row = D >> 3, total = (p.hi - p.lo) * per_row;
    for (int i = threadIdx.x; i < total; i += kBlock) {
      const int t = i / per_row, d = (i - t * per_row) * 8;
      const v2i w = *reinterpret_cast<const v2i*>(codes + (p.lo + t) * D + d);
      f32x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = there ? byte_of(w[e >> 2], e & 3) * scale : 0.0f;
      E::store8(out + t * ts + d, v);
    }
  } else {
    const int quads = D >> 2, g0 = p.lo >> 2, g1 = (p.hi + 3) >> 2;
    for (int i = threadIdx.x; i < (g1 - g0) * quads; i += kBlock) {
      const int grp = g0 + i / quads, d = (i % quads) * 4;
      const v4i w = *reinterpret_cast<const v4i*>(codes + (grp * D + d) * 4);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int place = 4 * grp + t;
        if (place < p.lo || place >= p.hi) continue;
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = there ? byte_of(w[e], t) * scale : 0.0f;
        E::store4(out + (place - p.lo) * ts + d, v);
      }
    }
  }
}

// workgroups of a call: pages that max_new rows of a sequence may touch, sequences, heads, keys and values
static int kv_grid(const mpq_kv_cache& c, const mpq_kv_batch& b, int threads, int64_t& pages_per_seq, dim3& grid) {
  const int64_t most = b.max_new < b.rows ? b.max_new : b.rows;
  pages_per_seq = (most + c.page - 2) / c.page + 1;
  if (pages_per_seq > b.table_pages) pages_per_seq = b.table_pages;
  int64_t want;
  if (__builtin_mul_overflow(pages_per_seq * b.seqs, (int64_t)2 * c.heads, &want) || want > ((int64_t)1 << 40)) return MPQ_ERR_SHAPE;
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
  const bool few = batch->max_new <= 2;
  int64_t pages;
  dim3 grid;
  rc = kv_grid(*cache, *batch, few ? kWave : kBlock, pages, grid);
  if (rc != MPQ_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
#define MPQ_APPEND(T_)                                                                                                       \
  (few ? (void)(kv_append_k<T_, kWave><<<grid, kWave, 0, st>>>(*cache, *batch, pages, k, k_token_stride, k_head_stride, v,   \
                                                               v_token_stride, v_head_stride))                               \
       : (void)(kv_append_k<T_, kBlock><<<grid, kBlock, 0, st>>>(*cache, *batch, pages, k, k_token_stride, k_head_stride, v, \
                                                                 v_token_stride, v_head_stride)))
  if (type == MPQ_F32) MPQ_APPEND(MPQ_F32);
  else if (type == MPQ_BF16) MPQ_APPEND(MPQ_BF16);
  else MPQ_APPEND(MPQ_F16);
#undef MPQ_APPEND
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
  dim3 grid;
  rc = kv_grid(*cache, *batch, kBlock, pages, grid);
  if (rc != MPQ_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (type == MPQ_F32) kv_gather_k<MPQ_F32><<<grid, kBlock, 0, st>>>(*cache, *batch, pages, k_out, v_out);
  else if (type == MPQ_BF16) kv_gather_k<MPQ_BF16><<<grid, kBlock, 0, st>>>(*cache, *batch, pages, k_out, v_out);
  else kv_gather_k<MPQ_F16><<<grid, kBlock, 0, st>>>(*cache, *batch, pages, k_out, v_out);
  return launch_status();
}
