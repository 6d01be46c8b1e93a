// The same for few rows over many keys: instances that take a share of the keys each, whose results are joined in layer_ops.cu.
#include "prompt_launch.h"

using namespace he;

int he::shares_error_count() {
  int n = 0;
  return cudaMemcpyFromSymbol(&n, he::g_tc_error, sizeof(int)) == cudaSuccess ? n : -1;
}

int he::launch_prompt_shares(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st) {
  return a.d <= 64 ? launch_prompt_tc<64, kOverShares>(a, maps, st) : launch_prompt_tc<128, kOverShares>(a, maps, st);
}
