// Host-side helpers that the library's translation units share: error text, argument checks, launches, tensor maps, and the
// launch of the attention over the cache.
#pragma once
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <mutex>
#include <utility>

#include "attend_kernels.cuh"
#include "common.cuh"
#include "device_table.h"
#include "hashevict.h"

#pragma GCC visibility push(hidden)

namespace he {

// The trouble counter (g_tc_error) of layer_ops.cu's kernels, -1 if it cannot be read.
int layer_error_count();

inline thread_local char g_err[512] = "";

inline int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}

#define HE_CUDA_CHECK(expr)                                                                         \
  do {                                                                                              \
    cudaError_t e_ = (expr);                                                                        \
    if (e_ != cudaSuccess) return fail(HE_ERR_CUDA, "%s failed: %s", #expr, cudaGetErrorString(e_)); \
  } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_config(const he_config* cfg, bool need_cache_dims) {
  if (cfg == nullptr) return fail(HE_ERR_INVALID_ARG, "cfg is null");
  if (cfg->dtype != HE_DTYPE_F32 && cfg->dtype != HE_DTYPE_BF16) return fail(HE_ERR_INVALID_ARG, "dtype %d is not HE_DTYPE_F32/BF16", cfg->dtype);
  if (cfg->hash_bits < 1 || cfg->hash_bits > 64) return fail(HE_ERR_INVALID_ARG, "hash_bits %d outside [1, 64]", cfg->hash_bits);
  if (cfg->head_dim < 8 || cfg->head_dim % 8 != 0) return fail(HE_ERR_INVALID_ARG, "head_dim %d is not a positive multiple of 8", cfg->head_dim);
  if (cfg->head_dim > kMaxDim) return fail(HE_ERR_UNSUPPORTED, "head_dim %d > %d", cfg->head_dim, kMaxDim);
  if (!need_cache_dims) return HE_OK;
  if (cfg->batch < 1 || cfg->n_kv_heads < 1) return fail(HE_ERR_INVALID_ARG, "batch %d / n_kv_heads %d must be >= 1", cfg->batch, cfg->n_kv_heads);
  if (cfg->group_size < 1) return fail(HE_ERR_INVALID_ARG, "group_size %d must be >= 1", cfg->group_size);
  if (cfg->group_size > kMaxGroup) return fail(HE_ERR_UNSUPPORTED, "group_size %d > %d", cfg->group_size, kMaxGroup);
  if (cfg->max_budget < 4 || cfg->max_budget % 4 != 0) return fail(HE_ERR_INVALID_ARG, "max_budget %d is not a positive multiple of 4", cfg->max_budget);
  if (cfg->max_budget > (1 << kKeyIdxBits)) return fail(HE_ERR_UNSUPPORTED, "max_budget %d > 2^20", cfg->max_budget);
  if (cfg->n_sink < 0 || cfg->n_recent < 0) return fail(HE_ERR_INVALID_ARG, "n_sink / n_recent must be >= 0");
  if (const int cb = packed_code_bytes(*cfg)) {
    if (cb > 3) return fail(HE_ERR_UNSUPPORTED, "packed codes of %d bytes per slot (hash_bits %d): 1 to 3, or whole words", cb, cfg->hash_bits);
    if (((long long)cfg->max_budget * cb) % 16 != 0)
      return fail(HE_ERR_INVALID_ARG, "packed codes: max_budget %d x %d bytes must be a multiple of 16", cfg->max_budget, cb);
  }
  return HE_OK;
}

inline int check_cache(const he_cache* ca) {
  if (ca == nullptr) return fail(HE_ERR_INVALID_ARG, "cache is null");
  if (!ca->k_cache || !ca->v_cache || !ca->codes || !ca->scores || !ca->pos || !ca->budget || !ca->fill || !ca->next_pos || !ca->W)
    return fail(HE_ERR_INVALID_ARG, "cache has a null pointer");
  if (!aligned16(ca->k_cache) || !aligned16(ca->v_cache) || !aligned16(ca->codes) || !aligned16(ca->scores) || !aligned16(ca->pos))
    return fail(HE_ERR_INVALID_ARG, "cache arrays must be 16-byte aligned");
  return HE_OK;
}

// Dynamic shared memory above the default limit needs a per-function opt-in; it is asked for once per
// (device, kernel) and again only if a larger size is needed.
template <typename K>
int set_smem(K kernel, size_t bytes) {
  // static + dynamic shared memory beyond 48 KB needs the opt-in, so ask whenever the sum could exceed it
  if (bytes <= 24 * 1024) return HE_OK;
  static std::mutex mu;
  static std::map<std::pair<int, const void*>, size_t> granted;
  int dev = 0;
  HE_CUDA_CHECK(cudaGetDevice(&dev));
  std::lock_guard<std::mutex> lock(mu);
  size_t& have = granted[std::make_pair(dev, reinterpret_cast<const void*>(kernel))];
  if (bytes > have) {
    HE_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    have = bytes;
  }
  return HE_OK;
}

// Decode launches carry the programmatic-serialization attribute so that consecutive he_decode_step kernels of a
// stream (or of a captured graph) overlap their launch latency; set HE_DISABLE_PDL=1 to launch them plainly.
inline bool pdl_enabled() {
  static const bool on = [] {
    const char* e = getenv("HE_DISABLE_PDL");
    return !(e && e[0] == '1');
  }();
  return on;
}

// Environment switches are read once per process (ID separates the call sites' caches).
template <int ID>
bool env_flag_set(const char* name) {
  static const bool on = getenv(name) != nullptr;
  return on;
}

// Launch with the programmatic-serialization attribute: the kernel may start while the stream's previous kernel still runs and
// calls griddepcontrol.wait before it touches anything that kernel or an earlier one may have written.
template <typename... P, typename... A>
int launch_pdl(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, bool pdl, cudaStream_t stream, A... args) {
  cudaLaunchConfig_t lc{};
  lc.gridDim = grid;
  lc.blockDim = dim3(threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = attr;
  lc.numAttrs = (pdl && pdl_enabled()) ? 1 : 0;
  HE_CUDA_CHECK(cudaLaunchKernelEx(&lc, kernel, args...));
  return HE_OK;
}

inline int sm_count(int* out) {
  static DeviceTable<1> table;
  int dev = 0;
  HE_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(HE_ERR_UNSUPPORTED, "device index %d", dev);
  return table.get(dev, 0, out, [dev](int* n) -> int {
    HE_CUDA_CHECK(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
    return HE_OK;
  });
}

// The driver's tensor-map encoder, or null.
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn tmap_encoder() {
  static EncodeTiledFn encode = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      fn = nullptr;
    return reinterpret_cast<EncodeTiledFn>(fn);
  }();
  return encode;
}

// Tensor map of a K or V cache [rows, d] in bf16: boxes of 64 channels x 32 rows, 128-byte swizzle. A map depends on the address
// and the shape alone, so the last few are kept per thread (a decode loop asks for the same ones at every token).
inline bool cache_rows_tmap(const void* base, long long rows, int d, CUtensorMap* out) {
  struct Entry {
    const void* base;
    long long rows;
    int d;
    CUtensorMap map;
  };
  constexpr int kEntries = 128;
  thread_local Entry cache[kEntries] = {};
  Entry& e = cache[(reinterpret_cast<uintptr_t>(base) >> 9) * 0x9E3779B97F4A7C15ull >> 57];
  if (e.base != base || e.rows != rows || e.d != d) {
    const EncodeTiledFn encode = tmap_encoder();
    if (encode == nullptr || rows > 0x7FFFFFFF || env_flag_set<3>("HE_DISABLE_TMA")) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)d * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)kAttendGroup}, estr[2] = {1, 1};
    if (encode(&e.map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
      e.base = nullptr;
      return false;
    }
    e.base = base, e.rows = rows, e.d = d;
  }
  *out = e.map;
  return true;
}

struct AttendMaps {
  alignas(64) CUtensorMap k, v;
};

template <int D, int NW, bool MOD, bool CAP, bool FOLD, bool BELOW>
int launch_attend_on(const AttendArgsOf<MOD>& a, const AttendMaps& maps, int S, size_t smem, cudaStream_t st) {
  if (int rc = set_smem(attend_bf16_kernel<D, NW, MOD, CAP, FOLD, BELOW>, smem)) return rc;
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3((unsigned)(a.cfg.n_kv_heads * S), (unsigned)a.cfg.batch);
  lc.blockDim = dim3(32 * NW);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)S;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = S > 1 ? 2 : 1;
  HE_CUDA_CHECK(cudaLaunchKernelEx(&lc, attend_bf16_kernel<D, NW, MOD, CAP, FOLD, BELOW>, a, S, maps.k, maps.v));
  return HE_OK;
}

// Dynamic shared memory of the attention kernel at most: a CTA's 227 KB less the mbarriers in static memory. One limit for every
// cluster size.
constexpr size_t kAttendMaxSmem = 227 * 1024 - 512;

template <int D>
constexpr size_t attend_smem(int S, int G) {
  return 1024 + (size_t)AttendRing<D, 8>::kBytes + (S > 1 ? (size_t)S * G * (D + 2) * sizeof(float) : 0);
}

// Tensor-core attention with S CTAs per unit. A call pays 2.5 us (one CTA) to 4 us (cluster of 8) whatever it reads, an SM pulls
// 90 GB/s, the GPU 6.3 TB/s, so a unit is spread until the grid has one CTA per SM. Measured (us per call in a graph, caches larger
// than L2; register-fed kernel with clusters of up to 8 before): 8 units of 9830 slots 16.9 -> 10.6, 32 of 2048 8.7 -> 7.9, 128 of
// 1024 14.6 -> 12.9.
template <int D, bool MOD, bool CAP = false, bool FOLD = false, bool BELOW = false>
int launch_attend(const AttendArgsOf<MOD>& a, const AttendMaps& maps, cudaStream_t st) {
  const long long units = (long long)a.cfg.batch * a.cfg.n_kv_heads;
  int sms = 0, dev = 0;
  if (int rc = sm_count(&sms)) return rc;
  HE_CUDA_CHECK(cudaGetDevice(&dev));
  static_assert(8 * kMaxGroup * (D + 2) * sizeof(float) <= AttendRing<D, 8>::kBytes, "the merge reuses the rings");
  static_assert(attend_smem<D>(8, kMaxGroup) <= kAttendMaxSmem, "up to eight CTAs any group's partial results fit");
  // As many CTAs per unit as keep the grid within one (deep) CTA per SM, and no fewer than 256 slots (a group per warp)
  // for each. Clusters above 8 need the driver's consent and as many free SMs in one GPC, so they are asked about.
  int S = (int)(sms / units < 16 ? sms / units : 16);
  if (S > a.cfg.max_budget / 256) S = a.cfg.max_budget / 256;
  if (S > 8) {
    static DeviceTable<17> table;  // clusters of S that the device holds at once (-1: none)
    for (S &= ~1; S > 8; S -= 2) {
      auto clusters_of = [S](int* got) -> int {
        cudaLaunchConfig_t oc{};
        oc.gridDim = dim3(S * 16);
        oc.blockDim = dim3(256);
        oc.dynamicSmemBytes = kAttendMaxSmem;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = S;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        oc.attrs = at;
        oc.numAttrs = 1;
        if (int rc = set_smem(attend_bf16_kernel<D, 8, MOD, CAP, FOLD, BELOW>, kAttendMaxSmem)) return rc;
        if (cudaFuncSetAttribute(attend_bf16_kernel<D, 8, MOD, CAP, FOLD, BELOW>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(got, attend_bf16_kernel<D, 8, MOD, CAP, FOLD, BELOW>, &oc) != cudaSuccess || *got < 1) {
          (void)cudaGetLastError();
          *got = -1;
        }
        return HE_OK;
      };
      int fit = 0;
      if (int rc = table.get(dev, S, &fit, clusters_of)) return rc;
      if (fit >= units && attend_smem<D>(S, a.cfg.group_size) <= kAttendMaxSmem) break;
    }
  }
  if (S < 1) S = 1;
  // Two small CTAs per SM once there are more units than SMs, so that one streams while the other starts or merges (512 units
  // of 1000 slots, d = 64: 24.4 against 27.7 us; level at 256 units of 2048 slots).
  if (units > sms) return launch_attend_on<D, 4, MOD, CAP, FOLD, BELOW>(a, maps, 1, 1024 + AttendRing<D, 4>::kBytes, st);
  return launch_attend_on<D, 8, MOD, CAP, FOLD, BELOW>(a, maps, S, attend_smem<D>(S, a.cfg.group_size), st);
}

}  // namespace he

#pragma GCC visibility pop
