// Attention of rows over keys of another length on the tensor cores (he_attend_cross): its instances of prompt_tc_kernel. A file of its own, as each compiles for a while.
#include "prompt_launch.h"

using namespace he;

int he::cross_error_count() {
  int n = 0;
  return cudaMemcpyFromSymbol(&n, he::g_tc_error, sizeof(int)) == cudaSuccess ? n : -1;
}

int he::launch_prompt_keys(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st) {
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  PromptArgs b = a;
  b.by_keys = a.batch > 1 && a.batch <= 32 && prompt_tc_tiles(a).items > sms;
  return a.d <= 64 ? launch_prompt_tc<64, kOverKeys>(b, maps, st) : launch_prompt_tc<128, kOverKeys>(b, maps, st);
}
