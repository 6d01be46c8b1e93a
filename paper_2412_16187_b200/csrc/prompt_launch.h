// Host side of the attention of prompts and of rows over keys of another length that layer_ops.cu, cross_ops.cu and cross_shares.cu share: tiles, tensor maps, launches.
#pragma once
#include "host_common.h"
#include "prompt_attend_kernels.cuh"

#pragma GCC visibility push(hidden)

namespace he {

// prompt_tc_kernel over keys of another length (cross_ops.cu), and with the keys shared out (cross_shares.cu): HE_OK, an error, or -1: the caller's other kernel serves.
int launch_prompt_keys(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st);
int launch_prompt_shares(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st);

// Few rows share a tile with those of the KV head's other query heads, 64 with a second one's, 32 with three others' (a warp's 32 rows are one head's). 3 sequences x 8 KV heads x 7
// heads of 5 rows over 6900 keys with a cap: 43 us, 167 without.
inline void prompt_pack(PromptArgs& a) {
  a.pack = 0, a.packs = a.group;
  if (a.self) return;
  while (a.pack < 2 && a.tokens <= kPtTile >> (a.pack + 1) && 1 << a.pack < a.group) ++a.pack;
  a.packs = (a.group + (1 << a.pack) - 1) >> a.pack;
}
// Work items of prompt_tc_kernel: two packs of query heads by a tile of rows, or one by two tiles.
struct PromptTiles {
  int by_heads, tiles;
  long long items;
};
inline PromptTiles prompt_tc_tiles(const PromptArgs& a) {
  PromptTiles t;
  t.by_heads = a.packs % 2 == 0;
  const int rows = (t.by_heads ? kPtTile : 2 * kPtTile) >> a.pack;
  t.tiles = (a.tokens + rows - 1) / rows;
  t.items = (long long)t.tiles * a.batch * a.n_kv_heads * a.packs / (t.by_heads ? 2 : 1);
  return t;
}
inline long long prompt_fp32_tiles(const PromptArgs& a, int rows) { return (long long)((a.tokens + rows - 1) / rows) * a.batch * a.n_kv_heads * a.group; }

// Tensor map of q, k or v: {channel, token, head, sequence} in boxes of 64 channels x 128 tokens (of several heads that many each), 128-byte swizzle. An axis of one
// entry may come with any stride, and gets one that the encoder takes.
inline bool prompt_tmap(const void* base, const PromptArgs& a, const long long strides[3], int heads, int tokens, int box_heads, CUtensorMap* out) {
  const EncodeTiledFn encode = tmap_encoder();
  if (encode == nullptr || env_flag_set<4>("HE_DISABLE_TMA")) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)a.d, (cuuint64_t)tokens, (cuuint64_t)heads, (cuuint64_t)a.batch};
  cuuint64_t st[3] = {(cuuint64_t)strides[2] * 2, (cuuint64_t)strides[1] * 2, (cuuint64_t)strides[0] * 2};
  for (int i = 0; i < 3; ++i) {
    if (dims[i + 1] == 1) st[i] = (cuuint64_t)a.d * 2;
    if (st[i] == 0 || st[i] % 16 != 0 || st[i] >= (1ull << 40)) return false;
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)(kPtTile / box_heads), (cuuint32_t)box_heads, 1}, estr[4] = {1, 1, 1, 1};
  return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, st, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether the kernel was built with as many registers a thread as its warps share out among themselves.
template <typename K>
int registers_suffice(K kernel, int* out) {
  cudaFuncAttributes at;
  HE_CUDA_CHECK(cudaFuncGetAttributes(&at, kernel));
  *out = at.numRegs * kPtThreads >= 256 * kPtSoftRegs + 128 * kPtOtherRegs ? 1 : 2;
  return HE_OK;
}

// HE_OK, an error, or -1: the caller's other kernel serves.
template <int D, bool CAP, bool BIAS, int KIND>
int launch_prompt_tc(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st) {
  auto kernel = prompt_tc_kernel<D, CAP, BIAS, KIND>;
  static DeviceTable<1> table;
  int dev = 0, enough = 0;
  HE_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(HE_ERR_UNSUPPORTED, "device index %d", dev);
  if (int rc = table.get(dev, 0, &enough, [&](int* got) { return registers_suffice(kernel, got); })) return rc;
  if (enough != 1) return -1;
  const PromptTiles t = prompt_tc_tiles(a);
  const long long ctas = t.items * (KIND == kOverShares ? a.splits : 1);
  if (ctas > 0x7FFFFFFFLL) return fail(HE_ERR_UNSUPPORTED, "%lld tiles in one call", ctas);
  if (int rc = set_smem(kernel, PromptTc<D>::kSmem)) return rc;
  return launch_pdl(kernel, dim3((unsigned)ctas), kPtThreads, PromptTc<D>::kSmem, true, st, a, t.tiles, t.by_heads, maps);
}
template <int D, int KIND>
int launch_prompt_tc(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st) {
  if (a.cap_log2 > 0.f)
    return a.slopes != nullptr ? launch_prompt_tc<D, true, true, KIND>(a, maps, st) : launch_prompt_tc<D, true, false, KIND>(a, maps, st);
  return a.slopes != nullptr ? launch_prompt_tc<D, false, true, KIND>(a, maps, st) : launch_prompt_tc<D, false, false, KIND>(a, maps, st);
}

}  // namespace he

#pragma GCC visibility pop
