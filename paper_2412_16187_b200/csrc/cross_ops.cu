// Attention of few rows over many keys on the tensor cores: the instances of prompt_tc_kernel that take a share of the keys each (he_attend_cross; their
// results are joined in layer_ops.cu). A file of its own, as each instance compiles for a while.
#include "prompt_launch.h"

using namespace he;

int he::cross_error_count() {
  int n = 0;
  return cudaMemcpyFromSymbol(&n, he::g_tc_error, sizeof(int)) == cudaSuccess ? n : -1;
}

int he::launch_prompt_shares(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st) {
  return a.d <= 64 ? launch_prompt_tc<64, true>(a, maps, st) : launch_prompt_tc<128, true>(a, maps, st);
}
