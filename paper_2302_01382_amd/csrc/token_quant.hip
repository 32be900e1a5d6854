// token_quant.hip -- Eq. 1 with a step per token (row): the row's maximum, its step size and its codes from one read.
//
// scale = fl32(m / qmax), inv = fl32(qmax / m), code = RNE(x * inv); |x| <= m, so that no code needs the clamp (|x * inv| <=
// qmax (1 + 2^-24)).  The row stays in registers between the maximum and the codes: K (el + 1) bytes per row travel, and
// that is what bounds a large call; a small one is two dependent memory latencies and a launch.
#include "types.hpp"

namespace mpq {

typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

__device__ __forceinline__ float magic(float x, float inv) { return __builtin_fmaf(x, inv, kMagic); }

// TPR: threads per row (a wave, or the workgroup); NCH: chunks of eight values that a thread holds, the rest of a longer
// row is read a second time (out of the L2).
template <int T, int TPR, int NCH>
__global__ __launch_bounds__(kBlock) void token_quant_k(const void* __restrict__ xv, int64_t M, int64_t K, int64_t stride, int bits,
                                                        int8_t* __restrict__ codes, float* __restrict__ scale_out) {
  using E = Elem<T>;
  typedef typename E::type El;
  constexpr int ROWS = kBlock / TPR;
  __shared__ float sm[kBlock / kWave];
  const int64_t row = block_index() * ROWS + (int)threadIdx.x / TPR;
  if (row >= M) return;  // uniform over the row's threads
  const El* x = reinterpret_cast<const El*>(xv) + row * stride;
  const int t = (int)threadIdx.x % TPR;
  const int64_t whole = K >> 3;
  f32x8 v[NCH];
  float m = 0.0f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int64_t i = t + c * TPR;
    v[c] = i < whole ? E::load8(x + 8 * i) : f32x8{0, 0, 0, 0, 0, 0, 0, 0};
  }
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[c][e]));
  for (int64_t i = t + NCH * TPR; i < whole; i += TPR) {
    const f32x8 w = E::load8(x + 8 * i);
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(w[e]));
  }
  const int64_t tail = 8 * whole + t;  // at most seven values behind the last chunk
  const float last = t < 8 && tail < K ? (float)x[tail] : 0.0f;
  m = wave_max(fmaxf(m, fabsf(last)));
  if (TPR > kWave) {
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  }
  float scale, inv;
  step_constants(m, bits, scale, inv);
  if (t == 0) scale_out[row] = scale;
  int8_t* out = codes + row * K;
  auto emit = [&](int64_t i, const f32x8& w) {
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = magic(w[e], inv);
    *reinterpret_cast<u32x2_any*>(out + 8 * i) = u32x2_any{low_bytes(q[0], q[1], q[2], q[3]), low_bytes(q[4], q[5], q[6], q[7])};
  };
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int64_t i = t + c * TPR;
    if (i < whole) emit(i, v[c]);
  }
  for (int64_t i = t + NCH * TPR; i < whole; i += TPR) emit(i, E::load8(x + 8 * i));
  if (t < 8 && tail < K) out[tail] = (int8_t)(bits_from_f(magic(last, inv)) & 0xFF);
}

int check_token_quant(const void* x, int x_type, int64_t M, int64_t K, int64_t x_stride, int bits) {
  if (M < 0 || K <= 0 || !known_type(x_type) || x_stride < K) return MPQ_ERR_SHAPE;
  if (mul_overflows(M, x_stride)) return MPQ_ERR_SHAPE;
  if (bits < 2 || bits > 8) return MPQ_ERR_BITS;
  if (M > 0 && !x) return MPQ_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(x) & (uintptr_t)(type_size(x_type) - 1)) return MPQ_ERR_ALIGN;
  return MPQ_OK;
}

int launch_token_quant(const void* x, int x_type, int64_t M, int64_t K, int64_t x_stride, int bits, int8_t* codes, float* scale,
                       hipStream_t st) {
  const bool wave_per_row = M >= 512 && K <= 4096;
  const int64_t per_thread = (K + 8 * (wave_per_row ? 64 : kBlock) - 1) / (8 * (wave_per_row ? 64 : kBlock));
  const dim3 grid = wide_grid(wave_per_row ? (M + 3) / 4 : M, kBlock);
#define MPQ_TQ(T_, TPR_, NCH_) token_quant_k<T_, TPR_, NCH_><<<grid, kBlock, 0, st>>>(x, M, K, x_stride, bits, codes, scale)
#define MPQ_TQ_T(T_)                                                                       \
  (wave_per_row ? (per_thread <= 2 ? (void)MPQ_TQ(T_, 64, 2) : (void)MPQ_TQ(T_, 64, 8))    \
                : (per_thread <= 2 ? (void)MPQ_TQ(T_, 256, 2) : (void)MPQ_TQ(T_, 256, 8)))
  if (x_type == MPQ_F32) MPQ_TQ_T(MPQ_F32);
  else if (x_type == MPQ_BF16) MPQ_TQ_T(MPQ_BF16);
  else MPQ_TQ_T(MPQ_F16);
#undef MPQ_TQ_T
#undef MPQ_TQ
  return launch_status();
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_token_quant(const void* x, int x_type, int64_t M, int64_t K, int64_t x_stride, int bits, int8_t* codes_out,
                               float* scale_out, void* stream) {
  const int rc = check_token_quant(x, x_type, M, K, x_stride, bits);
  if (rc != MPQ_OK) return rc;
  if (reinterpret_cast<uintptr_t>(scale_out) & 3u) return MPQ_ERR_ALIGN;
  if (M == 0) return MPQ_OK;
  if (!codes_out || !scale_out) return MPQ_ERR_NULL;
  return launch_token_quant(x, x_type, M, K, x_stride, bits, codes_out, scale_out, (hipStream_t)stream);
}
