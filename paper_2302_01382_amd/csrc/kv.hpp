// kv.hpp -- the key/value cache of quantized pages: what its calls share.
#pragma once

#include "types.hpp"

namespace mpq {

// argument checks of the three calls but for their own tensors
int check_kv(const mpq_kv_cache* c, const mpq_kv_batch* b, int type);

#if defined(__HIPCC__)

constexpr int64_t kMostTokens = 0x7FFFF000;  // of a sequence: a token's number and a few steps keep within 31 bits

// A sequence of a call.  Device arrays may hold anything: ranges are cut to the call's rows and to the table.
struct Sequence {
  int64_t row0;  // first row
  int n;         // rows
  int64_t len;   // tokens, the rows included; rows start at position len - n, which may be negative: those are absent
  int64_t room;  // tokens that the table has places for
};
__device__ __forceinline__ Sequence sequence(const mpq_kv_batch& b, int page, int s) {
  const int64_t rows = b.rows;
  int64_t s0 = b.starts[s], s1 = b.starts[s + 1];
  s0 = s0 < 0 ? 0 : s0 > rows ? rows : s0;
  s1 = s1 < s0 ? s0 : s1 > rows ? rows : s1;
  const int len = b.kv_len[s];
  Sequence q;
  q.row0 = s0;
  q.n = (int)(s1 - s0);
  q.len = len < 0 ? 0 : len;
  const int64_t room = (int64_t)b.table_pages * page;
  q.room = room < kMostTokens ? room : kMostTokens;
  return q;
}

#endif

}  // namespace mpq
