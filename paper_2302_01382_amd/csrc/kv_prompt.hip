// kv_prompt.hip -- the kernel and the launch of a prompt's attention (kv_prompt.hpp).
#include "kv_prompt.hpp"

namespace mpq {

template <int T, int DH, int NQ, bool ONE>
__global__ __launch_bounds__((PromptCfg<T, DH, NQ>::THREADS), DH == 4 ? 1 : 2) void kv_prompt_k(AttnArgs a, int64_t wg_tiles) {
  prompt_rows_body<T, DH, NQ, ONE, false>(a, wg_tiles, TreeMask{});
}

struct PromptKernels {
  typedef void (*Kern)(AttnArgs, int64_t);
  template <int T, int DH, int NQ>
  using Cfg = PromptCfg<T, DH, NQ>;
  template <int T, int DH, int NQ, bool ONE>
  static Kern kernel() { return kv_prompt_k<T, DH, NQ, ONE>; }
  static int launch(Kern k, dim3 grid, int threads, int lds, hipStream_t st, const AttnArgs& a, int64_t wg_tiles) {
    k<<<grid, threads, lds, st>>>(a, wg_tiles);
    return launch_status();
  }
};

// as many row tiles per wave as the registers hold
int prompt_rows(int type, int dim) { return type == MPQ_F32 && dim > 64 && dim <= 128 ? 64 : 128; }

int launch_prompt(int type, const AttnArgs& a, int64_t wg_tiles, int wg_rows, bool prepare_only, hipStream_t st) {
  return prompt_launch(PromptKernels{}, type, a, wg_tiles, wg_rows, prepare_only, st);
}

int prepare_prompt() { return prompt_prepare<PromptKernels>(); }

}  // namespace mpq
