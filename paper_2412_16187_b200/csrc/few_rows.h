// Few rows over many keys (he_attend_cross in layer_ops.cu) by the kernel of a new token's attention (pages.cu).
#pragma once
#include "host_common.h"

#pragma GCC visibility push(hidden)

namespace he {

struct RowsOverCall {
  const void *q, *k, *v;
  void* out;
  const int64_t *q_strides, *kv_strides, *out_strides;
  const int32_t *q_len, *kv_len, *q_pos, *first_key;
  const float* slopes;
  float* part;
  float scale_log2, cap_log2, inv_cap;
  int window, rows, keys;
};

// Whether units, a sequence's groups of 32 keys and a CTA's share of all of them can be counted in 32 bits (page_attend_kernel).
inline bool page_line_fits(const he_config* cfg, long long keys) {
  const double units = (double)cfg->batch * cfg->n_kv_heads, groups = (double)(keys / 32 + 1);
  return units < 2147483647.0 && (double)cfg->n_kv_heads * groups < 2147483647.0 && units * groups < 1e11;
}
// Whether `rows` rows of each query head over up to `keys` keys are few enough, where all rows of a sequence see the same keys.
inline bool few_rows(const he_config* cfg, int rows, int keys) {
  return cfg->dtype == HE_DTYPE_BF16 && cfg->head_dim <= 128 && keys > 0 && (long long)rows * cfg->group_size <= kMaxGroup &&
         page_line_fits(cfg, keys) && getenv("HE_DISABLE_ATTEND_MMA") == nullptr;
}
// Bytes of `part` (0: not served).
size_t few_rows_workspace(const he_config* cfg, int rows, int keys);
// HE_OK, an error, or -1: another kernel serves.
int launch_few_rows(const he_config* cfg, const RowsOverCall& call, cudaStream_t st);

}  // namespace he

#pragma GCC visibility pop
