// What a decoder layer does around the compressed cache: rotary positions of the rows that enter it (rotary_kernels.cuh), attention of the
// prompt over itself (prompt_attend_kernels.cuh) and the scored form of the attention over the cache (attend_kernels.cuh). Host side of these calls.
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>

#include "attend_kernels.cuh"
#include "common.cuh"
#include "hashevict.h"
#include "host_common.h"
#include "prompt_attend_kernels.cuh"
#include "rotary_kernels.cuh"

using namespace he;

int he::layer_error_count() {
  int n = 0;
  return cudaMemcpyFromSymbol(&n, he::g_tc_error, sizeof(int)) == cudaSuccess ? n : -1;
}

namespace {

constexpr int kMaxTokens = 1 << 24;  // positions and distances are exact in fp32

int check_rotary(const he_rotary* r, int d) {
  if (r == nullptr) return fail(HE_ERR_INVALID_ARG, "rotary is null");
  if (r->channels < 2 || r->channels % 2 != 0 || r->channels > 2 * HE_ROTARY_MAX_PAIRS)
    return fail(HE_ERR_INVALID_ARG, "rotary channels %d are not even and in [2, %d]", r->channels, 2 * HE_ROTARY_MAX_PAIRS);
  if (d > 0 && r->channels > d) return fail(HE_ERR_INVALID_ARG, "rotary channels %d > head_dim %d", r->channels, d);
  return HE_OK;
}

// Element strides of 16-byte aligned rows.
int check_strides(const char* what, const int64_t* strides, int n, int esize) {
  if (strides == nullptr) return fail(HE_ERR_INVALID_ARG, "%s strides are null", what);
  for (int i = 0; i < n; ++i)
    if (strides[i] < 0 || (strides[i] * esize) % 16 != 0)
      return fail(HE_ERR_INVALID_ARG, "%s stride %lld does not keep rows 16-byte aligned", what, (long long)strides[i]);
  return HE_OK;
}

// The rows of an output do not overlap: each axis of more than one entry steps over all that the axes of smaller strides cover. (n <= 3)
int check_apart(const char* what, const int64_t* strides, const long long* sizes, int n, int d) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + n, [&](int x, int y) { return strides[x] < strides[y]; });
  double covered = d;  // (exact as far as addresses go)
  for (int i = 0; i < n; ++i) {
    const int x = order[i];
    if (sizes[x] <= 1) continue;
    if ((double)strides[x] < covered) return fail(HE_ERR_INVALID_ARG, "%s stride %lld lets rows overlap", what, (long long)strides[x]);
    covered += (double)strides[x] * (double)(sizes[x] - 1);
  }
  return HE_OK;
}

template <int E, int V, bool INTER>
int launch_rotate_as(const RotateArgs& a, const he_rotary& r, dim3 grid, cudaStream_t st) {
  return launch_pdl(rotate_kernel<E, V, INTER>, grid, kRotateThreads, 0, true, st, a, r);
}

int launch_rotate(RotateArgs a, const he_rotary& r, cudaStream_t st) {
  const int es = esize_of(a.dtype), v = rotary_piece(r, es);
  a.units = rotary_units(r, a.d, v);
  const long long items = (long long)a.batch * a.tokens * a.units, blocks = (items + kRotateThreads - 1) / kRotateThreads;
  const int all = a.heads[0] + a.heads[1];
  if (blocks == 0 || all == 0) return HE_OK;
  if (blocks > 0x7FFFFFFFLL) return fail(HE_ERR_UNSUPPORTED, "%lld rows in one call", (long long)a.batch * a.tokens);
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  // Heads are shared out until there are enough CTAs for every SM, but a thread that has worked out its sines keeps at least four rows.
  const long long shares = (8LL * sms + blocks - 1) / blocks;
  a.heads_per_thread = (int)((all + shares - 1) / shares);
  if (a.heads_per_thread < 4) a.heads_per_thread = 4;
  if (a.next_pos != nullptr) a.heads_per_thread = 1;  // (each head's unit has a position of its own)
  if (a.heads_per_thread > all) a.heads_per_thread = all;
  const dim3 grid((unsigned)blocks, (unsigned)((all + a.heads_per_thread - 1) / a.heads_per_thread));
  if (grid.y > 65535) return fail(HE_ERR_UNSUPPORTED, "%d heads in one call", all);
  if (es == 2) {
    if (r.interleaved) return launch_rotate_as<2, 8, true>(a, r, grid, st);
    switch (v) {
      case 8: return launch_rotate_as<2, 8, false>(a, r, grid, st);
      case 4: return launch_rotate_as<2, 4, false>(a, r, grid, st);
      case 2: return launch_rotate_as<2, 2, false>(a, r, grid, st);
      default: return launch_rotate_as<2, 1, false>(a, r, grid, st);
    }
  }
  if (r.interleaved) return launch_rotate_as<4, 4, true>(a, r, grid, st);
  switch (v) {
    case 4: return launch_rotate_as<4, 4, false>(a, r, grid, st);
    case 2: return launch_rotate_as<4, 2, false>(a, r, grid, st);
    default: return launch_rotate_as<4, 1, false>(a, r, grid, st);
  }
}

// q and k of a rotation: each given with its output, or not at all.
int rotate_sides(RotateArgs& a, const he_config* cfg, const void* q, const void* k, void* q_out, void* k_out, const int64_t* const strides[4], int n,
                 long long tokens) {
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const int heads[2] = {cfg->n_kv_heads * cfg->group_size, cfg->n_kv_heads};
  for (int w = 0; w < 2; ++w) {
    const char* what = w ? "k" : "q";
    a.heads[w] = 0;
    if (in[w] == nullptr && out[w] == nullptr) continue;
    if (in[w] == nullptr || out[w] == nullptr || !aligned16(in[w]) || !aligned16(out[w]))
      return fail(HE_ERR_INVALID_ARG, "%s or its output is null or not 16-byte aligned", what);
    if (int rc = check_strides(what, strides[w], n, esize_of(cfg->dtype))) return rc;
    if (int rc = check_strides(w ? "k_out" : "q_out", strides[2 + w], n, esize_of(cfg->dtype))) return rc;
    const long long sizes[3] = {cfg->batch, heads[w], tokens};
    if (int rc = check_apart(w ? "k_out" : "q_out", strides[2 + w], sizes, n, cfg->head_dim)) return rc;
    a.x[w] = in[w], a.y[w] = out[w], a.heads[w] = heads[w];
    for (int i = 0; i < n; ++i) a.in[w][i] = strides[w][i], a.out[w][i] = strides[2 + w][i];
    if (in[w] == out[w])
      for (int i = 0; i < n; ++i)
        if (a.in[w][i] != a.out[w][i]) return fail(HE_ERR_INVALID_ARG, "%s is rotated in place with other strides", what);
  }
  if (a.heads[0] > 0 && a.heads[1] > 0 && (q_out == k_out || q_out == k || k_out == q))
    return fail(HE_ERR_INVALID_ARG, "q_out and k_out overlap each other or the other's input");
  return HE_OK;
}

// he_score_mod with its defaults filled in: the factor of q.k in log2 units and, with a cap, its two factors.
int check_mod(const he_score_mod* mod, int d, float* scale_log2, float* cap_log2, float* inv_cap, int* window, const float** slopes) {
  float scale = 1.0f / std::sqrt((float)d), cap = 0.f;
  *window = 0, *slopes = nullptr;
  if (mod != nullptr) {
    if (!(mod->scale >= 0.f) || std::isinf(mod->scale)) return fail(HE_ERR_INVALID_ARG, "scale %g is not finite and >= 0", (double)mod->scale);
    if (!(mod->cap >= 0.f) || std::isinf(mod->cap)) return fail(HE_ERR_INVALID_ARG, "cap %g is not finite and >= 0", (double)mod->cap);
    if (mod->window < 0) return fail(HE_ERR_INVALID_ARG, "window %d < 0", mod->window);
    if (mod->scale > 0.f) scale = mod->scale;
    cap = mod->cap, *window = mod->window, *slopes = mod->slopes;
  }
  *scale_log2 = scale * kLog2e, *cap_log2 = cap * kLog2e, *inv_cap = cap > 0.f ? scale / cap : 0.f;
  // (a ratio below the normal numbers would be lost, or its inverse: such a cap is none)
  if (!std::isfinite(*scale_log2) || !std::isfinite(*cap_log2) || !std::isfinite(*inv_cap) || (cap > 0.f && *inv_cap < FLT_MIN))
    return fail(HE_ERR_INVALID_ARG, "scale %g with cap %g leaves fp32", (double)scale, (double)cap);
  return HE_OK;
}

template <int NQ, int R>
int launch_prompt_fp32(const PromptArgs& a, cudaStream_t st) {
  const int tiles = (a.tokens + 16 * R - 1) / (16 * R);
  const long long ctas = (long long)tiles * a.batch * a.n_kv_heads * a.group;
  if (ctas > 0x7FFFFFFFLL) return fail(HE_ERR_UNSUPPORTED, "%lld tiles in one call", ctas);
  // a tile of keys ahead where an SM has one CTA and its 227 KB
  const int stages = R == 1 && a.dtype == HE_DTYPE_F32 && prompt_fp32_smem<R>(a.d, 2) <= kAttendMaxSmem ? 2 : 1;
  const size_t smem = prompt_fp32_smem<R>(a.d, stages);
  auto kernel = prompt_fp32_kernel<NQ, R>;
  if (int rc = set_smem(kernel, smem)) return rc;
  return launch_pdl(kernel, dim3((unsigned)ctas), kPromptThreads, smem, true, st, a, tiles, stages);
}
// Tiles of 64 rows once there is one for every SM, else of 16.
template <int NQ>
int launch_prompt_fp32(const PromptArgs& a, cudaStream_t st) {
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  const long long large = (long long)((a.tokens + 63) / 64) * a.batch * a.n_kv_heads * a.group;
  return large >= sms ? launch_prompt_fp32<NQ, 4>(a, st) : launch_prompt_fp32<NQ, 1>(a, st);
}

// Tensor map of q, k or v: {channel, token, head, sequence} in boxes of 64 channels x 128 tokens, 128-byte swizzle. An axis of one
// entry may come with any stride, and gets one that the encoder takes.
bool prompt_tmap(const void* base, const PromptArgs& a, const long long strides[3], int heads, CUtensorMap* out) {
  const EncodeTiledFn encode = tmap_encoder();
  if (encode == nullptr || env_flag_set<4>("HE_DISABLE_TMA")) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)a.d, (cuuint64_t)a.tokens, (cuuint64_t)heads, (cuuint64_t)a.batch};
  cuuint64_t st[3] = {(cuuint64_t)strides[2] * 2, (cuuint64_t)strides[1] * 2, (cuuint64_t)strides[0] * 2};
  for (int i = 0; i < 3; ++i) {
    if (dims[i + 1] == 1) st[i] = (cuuint64_t)a.d * 2;
    if (st[i] == 0 || st[i] % 16 != 0 || st[i] >= (1ull << 40)) return false;
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)kPtTile, 1, 1}, estr[4] = {1, 1, 1, 1};
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
template <int D, bool CAP, bool BIAS>
int launch_prompt_tc(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st) {
  auto kernel = prompt_tc_kernel<D, CAP, BIAS>;
  static DeviceTable<1> table;
  int dev = 0, enough = 0;
  HE_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(HE_ERR_UNSUPPORTED, "device index %d", dev);
  if (int rc = table.get(dev, 0, &enough, [&](int* got) { return registers_suffice(kernel, got); })) return rc;
  if (enough != 1) return -1;
  const int by_heads = a.group % 2 == 0, rows = by_heads ? kPtTile : 2 * kPtTile, tiles = (a.tokens + rows - 1) / rows;
  const long long ctas = (long long)tiles * a.batch * a.n_kv_heads * a.group / (by_heads ? 2 : 1);
  if (ctas > 0x7FFFFFFFLL) return fail(HE_ERR_UNSUPPORTED, "%lld tiles in one call", ctas);
  if (int rc = set_smem(kernel, PromptTc<D>::kSmem)) return rc;
  return launch_pdl(kernel, dim3((unsigned)ctas), kPtThreads, PromptTc<D>::kSmem, true, st, a, tiles, by_heads, maps);
}
template <int D>
int launch_prompt_tc(const PromptArgs& a, const PromptMaps& maps, cudaStream_t st) {
  if (a.cap_log2 > 0.f) return a.slopes != nullptr ? launch_prompt_tc<D, true, true>(a, maps, st) : launch_prompt_tc<D, true, false>(a, maps, st);
  return a.slopes != nullptr ? launch_prompt_tc<D, false, true>(a, maps, st) : launch_prompt_tc<D, false, false>(a, maps, st);
}

// Units that do not all run at once (two CTAs an SM) end evenly when the longest start first: 512 of 512 to 4096 slots 94 -> 85 us back to back. Known from the caller's mirror of the budgets; sorted again only when its contents
// change. A unit's result does not depend on it.
int order_units(ScoredArgs* a) {
  const int n = a->cfg.batch;
  const int32_t* budget = a->ca.budget_host;
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  a->n_order = 0;
  if (budget == nullptr || n > 256 || (long long)n * a->cfg.n_kv_heads <= 2 * sms) return HE_OK;
  struct Order {
    int n = 0;
    int32_t budget[256];
    uint8_t order[256];
  };
  thread_local Order known;
  if (known.n != n || memcmp(known.budget, budget, sizeof(int32_t) * n) != 0) {
    known.n = n;
    memcpy(known.budget, budget, sizeof(int32_t) * n);
    for (int i = 0; i < n; ++i) known.order[i] = (uint8_t)i;
    std::stable_sort(known.order, known.order + n, [&](uint8_t x, uint8_t y) { return known.budget[x] > known.budget[y]; });
  }
  a->n_order = n;
  memcpy(a->order, known.order, n);
  return HE_OK;
}

template <bool CAP, bool FOLD>
int launch_scored_bf16(const ScoredArgs& a, const AttendMaps& maps, cudaStream_t st) {
  switch (a.cfg.head_dim) {
    case 64: return launch_attend<64, true, CAP, FOLD, false>(a, maps, st);
    case 128: return launch_attend<128, true, CAP, FOLD, false>(a, maps, st);
    default: return a.cfg.head_dim < 64 ? launch_attend<64, true, CAP, FOLD, true>(a, maps, st) : launch_attend<128, true, CAP, FOLD, true>(a, maps, st);
  }
}

// As many CTAs per unit as keep the grid within two per SM, at most 8 (a cluster of any device) and no fewer than two tiles of slots for each.
template <int E, int GP>
int launch_scored(const ScoredArgs& a, cudaStream_t st) {
  const long long units = (long long)a.cfg.batch * a.cfg.n_kv_heads;
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  int S = 1;
  while (S < 8 && 2 * S * units <= 2 * sms && 2 * S * 2 * kScoredSlots <= a.cfg.max_budget) S *= 2;
  // a tile ahead where an SM has one CTA and its 227 KB
  const int stages = E == 4 && S * units <= sms && scored_smem(S, 2, a.cfg.group_size, a.cfg.head_dim) <= kAttendMaxSmem ? 2 : 1;
  const size_t smem = scored_smem(S, stages, a.cfg.group_size, a.cfg.head_dim);
  auto kernel = attend_scored_kernel<E, GP>;
  if (int rc = set_smem(kernel, smem)) return rc;
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3((unsigned)(a.cfg.n_kv_heads * S), (unsigned)a.cfg.batch);
  lc.blockDim = dim3(kAttendThreads);
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
  HE_CUDA_CHECK(cudaLaunchKernelEx(&lc, kernel, a, S, stages));
  return HE_OK;
}

}  // namespace

extern "C" {

int he_rotary_init_frequencies(he_rotary* out, int32_t channels, int32_t interleaved, const double* frequencies, double amplitude) {
  if (out == nullptr || frequencies == nullptr) return fail(HE_ERR_INVALID_ARG, "out or frequencies is null");
  he_rotary r{};
  r.channels = channels, r.interleaved = interleaved != 0;
  if (int rc = check_rotary(&r, 0)) return rc;
  if (!std::isfinite(amplitude) || !std::isfinite((float)amplitude)) return fail(HE_ERR_INVALID_ARG, "amplitude %g is not finite", amplitude);
  r.amplitude = (float)amplitude;
  const long double two_pi = 8.0L * atanl(1.0L);
  for (int i = 0; i < channels / 2; ++i) {
    if (!std::isfinite(frequencies[i])) return fail(HE_ERR_INVALID_ARG, "frequency %d is not finite", i);
    long double t = (long double)frequencies[i] / two_pi;
    t -= floorl(t);                            // turns modulo 1
    const long double scaled = ldexpl(t, 64);  // (a turn that rounds up to 2^64 is none)
    r.turns[i] = scaled >= 18446744073709551615.0L ? 0ull : (uint64_t)(scaled + 0.5L);
  }
  *out = r;
  return HE_OK;
}

int he_rotary_init(he_rotary* out, int32_t channels, int32_t interleaved, double base, int32_t stretch, double factor, double length,
                   double low, double high) {
  he_rotary r{};
  r.channels = channels;
  if (int rc = check_rotary(&r, 0)) return rc;
  if (!(base > 1.0) || !std::isfinite(base)) return fail(HE_ERR_INVALID_ARG, "base %g is not finite and > 1", base);
  if (stretch < HE_ROTARY_PLAIN || stretch > HE_ROTARY_BANDS) return fail(HE_ERR_INVALID_ARG, "stretch %d is unknown", stretch);
  if (stretch != HE_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return fail(HE_ERR_INVALID_ARG, "factor %g is not finite and >= 1", factor);
  if (stretch >= HE_ROTARY_YARN && (!(length > 0.0) || !std::isfinite(length) || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
    return fail(HE_ERR_INVALID_ARG, "length %g, low %g, high %g: 0 < length and 0 < low < high are needed", length, low, high);
  if (stretch == HE_ROTARY_NTK && channels == 2) return fail(HE_ERR_INVALID_ARG, "NTK needs more than one pair");
  const double two_pi = 2.0 * M_PI, rd = channels;
  double f[HE_ROTARY_MAX_PAIRS], amplitude = 1.0;
  if (stretch == HE_ROTARY_NTK) base *= std::pow(factor, rd / (rd - 2.0));
  // YARN: the pair index at which a pair makes n turns over `length` (a real number)
  auto pair_of = [&](double n) { return rd * std::log(length / (n * two_pi)) / (2.0 * std::log(base)); };
  const double first = stretch == HE_ROTARY_YARN ? std::fmax(std::floor(pair_of(high)), 0.0) : 0.0;
  const double last = stretch == HE_ROTARY_YARN ? std::fmin(std::ceil(pair_of(low)), rd - 1.0) : 0.0;
  for (int i = 0; i < channels / 2; ++i) {
    f[i] = std::pow(base, -2.0 * i / rd);
    double keep = 1.0;  // share of the frequency that is not stretched
    if (stretch == HE_ROTARY_LINEAR) keep = 0.0;
    if (stretch == HE_ROTARY_YARN) keep = 1.0 - std::fmin(std::fmax((i - first) / std::fmax(last - first, 0.001), 0.0), 1.0);
    if (stretch == HE_ROTARY_BANDS) keep = std::fmin(std::fmax((length * f[i] / two_pi - low) / (high - low), 0.0), 1.0);
    f[i] = keep * f[i] + (keep < 1.0 ? (1.0 - keep) * f[i] / factor : 0.0);
  }
  if (stretch == HE_ROTARY_YARN) amplitude = 0.1 * std::log(factor) + 1.0;
  return he_rotary_init_frequencies(out, channels, interleaved, f, amplitude);
}

int he_rotate_prompt(const he_config* cfg, const he_rotary* rotary, const void* q, const void* k, const int64_t q_strides[3],
                     const int64_t k_strides[3], const int32_t* positions, const int32_t* prompt_len, int32_t max_prompt_len, void* q_out,
                     void* k_out, const int64_t q_out_strides[3], const int64_t k_out_strides[3], void* stream) {
  if (int rc = check_config(cfg, true)) return rc;
  if (int rc = check_rotary(rotary, cfg->head_dim)) return rc;
  if (max_prompt_len < 0) return fail(HE_ERR_INVALID_ARG, "max_prompt_len %d < 0", max_prompt_len);
  if (max_prompt_len == 0) return HE_OK;
  RotateArgs a{};
  const int64_t* const strides[4] = {q_strides, k_strides, q_out_strides, k_out_strides};
  if (int rc = rotate_sides(a, cfg, q, k, q_out, k_out, strides, 3, max_prompt_len)) return rc;
  a.n_kv_heads = cfg->n_kv_heads, a.group = cfg->group_size, a.d = cfg->head_dim, a.dtype = cfg->dtype;
  a.batch = cfg->batch, a.tokens = max_prompt_len, a.positions = positions, a.lens = prompt_len;
  return launch_rotate(a, *rotary, static_cast<cudaStream_t>(stream));
}

int he_rotate_step(const he_config* cfg, const he_rotary* rotary, const he_cache* cache, const void* q, const void* k,
                   const int64_t q_strides[2], const int64_t k_strides[2], void* q_out, void* k_out, const int64_t q_out_strides[2],
                   const int64_t k_out_strides[2], void* stream) {
  if (int rc = check_config(cfg, true)) return rc;
  if (int rc = check_rotary(rotary, cfg->head_dim)) return rc;
  if (cache == nullptr || cache->next_pos == nullptr) return fail(HE_ERR_INVALID_ARG, "cache or its next_pos is null");
  // such a step reads its rows before the kernel ahead of it in the stream, this one, has written them
  if (cfg->flags & HE_FLAG_EARLY_INPUTS)
    return fail(HE_ERR_INVALID_ARG, "rows rotated for the next step are written too late for HE_FLAG_EARLY_INPUTS");
  RotateArgs a{};
  const int64_t* const strides[4] = {q_strides, k_strides, q_out_strides, k_out_strides};
  if (int rc = rotate_sides(a, cfg, q, k, q_out, k_out, strides, 2, 1)) return rc;
  a.n_kv_heads = cfg->n_kv_heads, a.group = cfg->group_size, a.d = cfg->head_dim, a.dtype = cfg->dtype;
  a.batch = cfg->batch, a.tokens = 1, a.next_pos = cache->next_pos;
  return launch_rotate(a, *rotary, static_cast<cudaStream_t>(stream));
}

int he_attend_prompt(const he_config* cfg, const he_score_mod* mod, const void* q, const void* k, const void* v, const int64_t q_strides[3],
                     const int64_t kv_strides[3], const int32_t* prompt_len, int32_t max_prompt_len, const int32_t* doc_start,
                     const int32_t* prefix_len, void* out, const int64_t out_strides[3], void* stream) {
  if (int rc = check_config(cfg, true)) return rc;
  if (max_prompt_len < 0) return fail(HE_ERR_INVALID_ARG, "max_prompt_len %d < 0", max_prompt_len);
  if (max_prompt_len > kMaxTokens) return fail(HE_ERR_UNSUPPORTED, "max_prompt_len %d > 2^24", max_prompt_len);
  PromptArgs a{};
  if (int rc = check_mod(mod, cfg->head_dim, &a.scale_log2, &a.cap_log2, &a.inv_cap, &a.window, &a.slopes)) return rc;
  a.near_end = a.inv_cap >= kPtNearInv && a.inv_cap <= kPtNearMost ? kPtNearEnd : -1.f;
  if (max_prompt_len == 0) return HE_OK;
  if (!q || !k || !v || !out || !prompt_len) return fail(HE_ERR_INVALID_ARG, "q, k, v, out or prompt_len is null");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return fail(HE_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned");
  const int es = esize_of(cfg->dtype);
  if (int rc = check_strides("q", q_strides, 3, es)) return rc;
  if (int rc = check_strides("k / v", kv_strides, 3, es)) return rc;
  if (int rc = check_strides("out", out_strides, 3, es)) return rc;
  const long long sizes[3] = {cfg->batch, (long long)cfg->n_kv_heads * cfg->group_size, max_prompt_len};
  if (int rc = check_apart("out", out_strides, sizes, 3, cfg->head_dim)) return rc;
  if (out == q || out == k || out == v) return fail(HE_ERR_INVALID_ARG, "out overlaps q, k or v");
  a.q = q, a.k = k, a.v = v, a.out = out;
  for (int i = 0; i < 3; ++i) a.qs[i] = q_strides[i], a.ks[i] = kv_strides[i], a.os[i] = out_strides[i];
  a.batch = cfg->batch, a.n_kv_heads = cfg->n_kv_heads, a.group = cfg->group_size, a.d = cfg->head_dim, a.dtype = cfg->dtype, a.tokens = max_prompt_len;
  a.lens = prompt_len, a.doc_start = doc_start, a.prefix = prefix_len;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a.dtype == HE_DTYPE_BF16 && a.d <= 128 && getenv("HE_DISABLE_ATTEND_MMA") == nullptr) {
    PromptMaps maps;
    if (prompt_tmap(q, a, a.qs, a.n_kv_heads * a.group, &maps.q) && prompt_tmap(k, a, a.ks, a.n_kv_heads, &maps.k) &&
        prompt_tmap(v, a, a.ks, a.n_kv_heads, &maps.v)) {
      const int rc = a.d <= 64 ? launch_prompt_tc<64>(a, maps, st) : launch_prompt_tc<128>(a, maps, st);
      if (rc >= 0) return rc;
    }
  }
  switch ((a.d + 63) / 64) {
    case 1: return launch_prompt_fp32<1>(a, st);
    case 2: return launch_prompt_fp32<2>(a, st);
    case 3: return launch_prompt_fp32<3>(a, st);
    default: return launch_prompt_fp32<4>(a, st);
  }
}

int he_attend_scored(const he_config* cfg, const he_cache* cache, const he_score_mod* mod, const void* q, const int32_t* first_pos, float* out,
                     void* stream) {
  if (int rc = check_config(cfg, true)) return rc;
  if (int rc = check_cache(cache)) return rc;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return fail(HE_ERR_INVALID_ARG, "q or out is null or not 16-byte aligned");
  if (cfg->batch > 65535) return fail(HE_ERR_UNSUPPORTED, "batch %d > 65535 in one call", cfg->batch);
  ScoredArgs a{{*cfg, *cache, q, out, {}}, 0, {}};
  const int G = cfg->group_size, d = cfg->head_dim;
  if (int rc = check_mod(mod, d, &a.mod.scale_log2, &a.mod.cap_log2, &a.mod.inv_cap, &a.mod.window, &a.mod.slopes)) return rc;
  a.mod.first_pos = first_pos;
  if (int rc = order_units(&a)) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cfg->dtype == HE_DTYPE_BF16 && d <= 128 && getenv("HE_DISABLE_ATTEND_MMA") == nullptr) {
    const long long rows = (long long)cfg->batch * cfg->n_kv_heads * cfg->max_budget;
    AttendMaps maps;
    if (cache_rows_tmap(cache->k_cache, rows, d, &maps.k) && cache_rows_tmap(cache->v_cache, rows, d, &maps.v))
      return a.mod.cap_log2 > 0.f ? (G <= 4 ? launch_scored_bf16<true, true>(a, maps, st) : launch_scored_bf16<true, false>(a, maps, st))
                                  : (G <= 4 ? launch_scored_bf16<false, true>(a, maps, st) : launch_scored_bf16<false, false>(a, maps, st));
  }
  if (G == 1) return cfg->dtype == HE_DTYPE_BF16 ? launch_scored<2, 1>(a, st) : launch_scored<4, 1>(a, st);
  if (G == 2) return cfg->dtype == HE_DTYPE_BF16 ? launch_scored<2, 2>(a, st) : launch_scored<4, 2>(a, st);
  if (G <= 4) return cfg->dtype == HE_DTYPE_BF16 ? launch_scored<2, 4>(a, st) : launch_scored<4, 4>(a, st);
  return cfg->dtype == HE_DTYPE_BF16 ? launch_scored<2, 8>(a, st) : launch_scored<4, 8>(a, st);
}

}  // extern "C"
