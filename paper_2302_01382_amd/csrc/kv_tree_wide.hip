// kv_tree_wide.hip -- attention of a tree of drafted tokens where a sequence brings many rows: the prompt's kernel (kv_prompt.hpp)
// with the tree's bits as its mask.  24 sequences of up to 13 drafted tokens behind up to 8000, 32 / 8 heads of 128 in bf16: 88 us in pieces of
// 64 rows, vector instructions 44 % and matrix steps 26 % of the cycles, 294 MB read (77 with one term of a probability, which leaves outputs
// 8.9e-4 of their norm from fp32 products in place of 8e-5); 61 behind 65500 in fp16: 117 in pieces of 128, 50 % and 37 %.
#include "kv_prompt.hpp"

namespace mpq {

constexpr bool kSingle(int dh, int nq) { return dh <= 2 && nq == 1; }
template <int T, int DH, int NQ, bool ONE>
__global__ __launch_bounds__((PromptCfg<T, DH, NQ>::THREADS), DH == 4 ? 1 : kSingle(DH, NQ) && T != MPQ_F32 ? 3 : 2) void kv_tree_wide_k(AttnArgs a, int64_t wg_tiles, TreeMask tree) {
  prompt_rows_body<T, DH, NQ, ONE, true, kSingle(DH, NQ)>(a, wg_tiles, tree);
}

struct TreeKernels {
  typedef void (*Kern)(AttnArgs, int64_t, TreeMask);
  template <int T, int DH, int NQ>
  using Cfg = PromptCfg<T, DH, NQ, kSingle(DH, NQ)>;
  TreeMask tree;
  template <int T, int DH, int NQ, bool ONE>
  static Kern kernel() { return kv_tree_wide_k<T, DH, NQ, ONE>; }
  int launch(Kern k, dim3 grid, int threads, int lds, hipStream_t st, const AttnArgs& a, int64_t wg_tiles) const {
    k<<<grid, threads, lds, st>>>(a, wg_tiles, tree);
    return launch_status();
  }
};

int launch_tree_wide(int type, const AttnArgs& a, const TreeMask& tree, int64_t wg_tiles, int wg_rows, hipStream_t st) {
  return prompt_launch(TreeKernels{tree}, type, a, wg_tiles, wg_rows, false, st);
}

int prepare_tree_wide() { return prompt_prepare<TreeKernels>(); }

}  // namespace mpq
