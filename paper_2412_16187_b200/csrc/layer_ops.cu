// What a decoder layer does around the compressed cache: rotary positions of the rows that enter it (rotary_kernels.cuh), attention of the
// prompt over itself (prompt_attend_kernels.cuh) and the scored form of the attention over the cache (attend_kernels.cuh). Host side of these calls.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "attend_kernels.cuh"
#include "common.cuh"
#include "few_rows.h"
#include "hashevict.h"
#include "host_common.h"
#include "prompt_attend_kernels.cuh"
#include "prompt_launch.h"
#include "rotary_kernels.cuh"

using namespace he;

int he::layer_error_count() {
  int n = 0;
  return cudaMemcpyFromSymbol(&n, he::g_tc_error, sizeof(int)) == cudaSuccess ? n : -1;
}

namespace {

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

template <int NQ, int R>
int launch_prompt_fp32(const PromptArgs& a, cudaStream_t st) {
  const int tiles = (a.tokens + 16 * R - 1) / (16 * R);
  const long long ctas = (long long)tiles * a.batch * a.n_kv_heads * a.group * a.splits;
  if (ctas > 0x7FFFFFFFLL) return fail(HE_ERR_UNSUPPORTED, "%lld tiles in one call", ctas);
  // a tile of keys ahead where an SM has one CTA and its 227 KB
  const int stages = R == 1 && a.dtype == HE_DTYPE_F32 && prompt_fp32_smem<R>(a.d, 2) <= kAttendMaxSmem ? 2 : 1;
  const size_t smem = prompt_fp32_smem<R>(a.d, stages);
  auto kernel = prompt_fp32_kernel<NQ, R>;
  if (int rc = set_smem(kernel, smem)) return rc;
  return launch_pdl(kernel, dim3((unsigned)ctas), kPromptThreads, smem, true, st, a, tiles, stages);
}
// Tiles of 64 rows once there is one for every SM, else of 16 (also for up to 16 rows over keys of another length).
template <int NQ>
int launch_prompt_fp32(const PromptArgs& a, cudaStream_t st) {
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  return prompt_fp32_tiles(a, 64) >= sms && (a.self || a.tokens > 16) ? launch_prompt_fp32<NQ, 4>(a, st) : launch_prompt_fp32<NQ, 1>(a, st);
}

bool on_tensor_cores(const PromptArgs& a) { return a.dtype == HE_DTYPE_BF16 && a.d <= 128 && getenv("HE_DISABLE_ATTEND_MMA") == nullptr; }

size_t prompt_part_bytes(const PromptArgs& a, int splits) {
  return splits > 1 ? (size_t)splits * a.batch * a.n_kv_heads * a.group * a.tokens * (a.d + 2) * sizeof(float) : 0;
}

// Into how many shares the keys are cut where there are fewer tiles of rows than SMs. Tiles run side by side on the SMs, in rounds; a block of 128 keys costs
// a tile 3500 cycles on the tensor cores and the tile's own start and end 9000 (prompt_tc_kernel), and each share of a row goes through HBM or L2 twice in fp32 (3400 bytes
// a cycle). So the best count is the one with the least of rounds, starts and traffic, all for the longest rows and keys of the call: 32 heads of 512 rows over 32768 keys 265 us
// with 2 shares, 483 with one, 327 with 9. On the CUDA cores a block of 64 keys by 16 or 64 rows takes the place.
constexpr int kMostShares = 64, kMostRounds = 8;  // of a tile; of tiles times shares, where there is more than one
// Tiles of rows, as many as run at once, blocks of keys.
struct PromptWork {
  long long items, blocks;
  int at_once;
};
int prompt_work(const PromptArgs& a, bool tc, PromptWork* w) {
  if (int rc = sm_count(&w->at_once)) return rc;
  if (!tc && a.d <= 128) w->at_once *= 2;  // (CTAs of an SM)
  w->items = tc ? prompt_tc_tiles(a).items : prompt_fp32_tiles(a, 64);
  if (!tc && (w->items < w->at_once || a.tokens <= 16)) w->items = prompt_fp32_tiles(a, 16);
  w->blocks = ((long long)a.keys + (tc ? 127 : 63)) / (tc ? 128 : 64);
  return HE_OK;
}
int prompt_splits(const PromptArgs& a, bool tc, int* out) {
  PromptWork w;
  if (int rc = prompt_work(a, tc, &w)) return rc;
  *out = 1;
  double best = 0.0;
  for (int z = 1; z <= kMostShares && 2 * z <= w.blocks && (z == 1 || w.items * z <= (long long)kMostRounds * w.at_once); ++z) {
    const double rounds = (double)((w.items * z + w.at_once - 1) / w.at_once), cost = rounds * ((double)((w.blocks + z - 1) / z) * 3500.0 + 9000.0) + (z > 1 ? 6000.0 + (double)prompt_part_bytes(a, z) * 2.0 / 3400.0 : 0.0);
    if (z == 1 || cost < 0.95 * best) best = cost, *out = z;
  }
  return HE_OK;
}
// Bytes that the shares of any call of up to a.tokens rows over up to a.keys keys fit in. Fewer rows may take more shares, and which of them a call takes is no simple function
// of its sizes; so this is what its limits allow: as many as the blocks of keys and the rounds leave for each count of tiles, which changes at multiples of 16 rows.
int prompt_most_bytes(PromptArgs a, bool tc, size_t* out) {
  const int tokens = a.tokens;
  *out = 0;
  for (int n = 16;; n += 16) {
    a.tokens = std::min(n, tokens);
    prompt_pack(a);
    PromptWork w;
    if (int rc = prompt_work(a, tc, &w)) return rc;
    const long long most = std::min<long long>({kMostShares, w.blocks / 2, (long long)kMostRounds * w.at_once / w.items});
    if (most > 1) *out = std::max(*out, prompt_part_bytes(a, (int)most));
    if (n >= tokens || (n > 64 && 2 * w.items > (long long)kMostRounds * w.at_once)) return HE_OK;  // (from 64 rows on tiles become more with the rows)
  }
}
int launch_rows(const PromptArgs& a, bool tc, cudaStream_t st) {
  if (tc) {
    PromptMaps maps;
    if (prompt_tmap(a.q, a, a.qs, a.n_kv_heads * a.group, a.tokens, 1 << a.pack, &maps.q) && prompt_tmap(a.k, a, a.ks, a.n_kv_heads, a.keys, 1, &maps.k) &&
        prompt_tmap(a.v, a, a.ks, a.n_kv_heads, a.keys, 1, &maps.v)) {
      const int rc = a.splits > 1 ? launch_prompt_shares(a, maps, st) : !a.self ? launch_prompt_keys(a, maps, st)
                     : a.d <= 64  ? launch_prompt_tc<64, kOverSelf>(a, maps, st) : launch_prompt_tc<128, kOverSelf>(a, maps, st);
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

// he_attend_prompt and he_attend_cross. `a` comes with lengths, positions and masks.
int attend_rows(PromptArgs& a, const he_config* cfg, const he_score_mod* mod, const void* q, const void* k, const void* v, const int64_t* q_strides,
                const int64_t* kv_strides, void* out, const int64_t* out_strides, const char* tokens_name, void* workspace, size_t workspace_bytes, cudaStream_t st) {
  if (int rc = check_config(cfg, true)) return rc;
  if (a.tokens < 0) return fail(HE_ERR_INVALID_ARG, "%s %d < 0", tokens_name, a.tokens);
  if (a.keys < 0) return fail(HE_ERR_INVALID_ARG, "max_kv_len %d < 0", a.keys);
  if (a.tokens > kMaxTokens) return fail(HE_ERR_UNSUPPORTED, "%s %d > 2^24", tokens_name, a.tokens);
  if (a.keys > kMaxTokens) return fail(HE_ERR_UNSUPPORTED, "max_kv_len %d > 2^24", a.keys);
  if (int rc = check_mod(mod, cfg->head_dim, &a.scale_log2, &a.cap_log2, &a.inv_cap, &a.window, &a.slopes)) return rc;
  a.near_end = a.inv_cap >= kPtNearInv && a.inv_cap <= kPtNearMost ? kPtNearEnd : -1.f;
  if (a.tokens == 0) return HE_OK;
  if (!q || !out || !a.lens || !a.kv_lens || (a.keys > 0 && (!k || !v))) return fail(HE_ERR_INVALID_ARG, "q, k, v, out or a length is null");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return fail(HE_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned");
  const int es = esize_of(cfg->dtype);
  if (int rc = check_strides("q", q_strides, 3, es)) return rc;
  if (int rc = check_strides("k / v", kv_strides, 3, es)) return rc;
  if (int rc = check_strides("out", out_strides, 3, es)) return rc;
  const long long sizes[3] = {cfg->batch, (long long)cfg->n_kv_heads * cfg->group_size, a.tokens};
  if (int rc = check_apart("out", out_strides, sizes, 3, cfg->head_dim)) return rc;
  if (out == q || (a.keys > 0 && (out == k || out == v))) return fail(HE_ERR_INVALID_ARG, "out overlaps q, k or v");
  a.q = q, a.k = k, a.v = v, a.out = out;
  for (int i = 0; i < 3; ++i) a.qs[i] = q_strides[i], a.ks[i] = kv_strides[i], a.os[i] = out_strides[i];
  a.batch = cfg->batch, a.n_kv_heads = cfg->n_kv_heads, a.group = cfg->group_size, a.d = cfg->head_dim, a.dtype = cfg->dtype;
  prompt_pack(a);
  const bool tc = on_tensor_cores(a);
  if (workspace != nullptr) {
    // one row a sequence, or a few that see the same keys: K and V are read once for all of them
    const size_t few = a.prefix == nullptr && (a.tokens == 1 || (a.all && a.doc_start == nullptr)) ? few_rows_workspace(cfg, a.tokens, a.keys) : 0;
    if (few > 0) {
      if (few > workspace_bytes) return fail(HE_ERR_WORKSPACE, "workspace of %zu bytes, %zu are needed", workspace_bytes, few);
      const RowsOverCall call{q, k, v, out, q_strides, kv_strides, out_strides, a.lens, a.kv_lens, a.q_pos, a.doc_start, a.slopes, static_cast<float*>(workspace),
                              a.scale_log2, a.cap_log2, a.inv_cap, a.window, a.tokens, a.keys};
      const int rc = launch_few_rows(cfg, call, st);
      if (rc >= 0) return rc;
    }
    if (int rc = prompt_splits(a, tc, &a.splits)) return rc;
    if (prompt_part_bytes(a, a.splits) > workspace_bytes)
      return fail(HE_ERR_WORKSPACE, "workspace of %zu bytes, %zu are needed", workspace_bytes, prompt_part_bytes(a, a.splits));
    a.part = static_cast<float*>(workspace);
  }
  if (a.keys == 0) a.splits = 1;
  const bool far = a.cap_log2 >= kPtFar && a.slopes == nullptr;  // (scores that prompt_tc_kernel with a cap has no form for)
  if (int rc = launch_rows(a, tc && a.keys > 0 && !far, st)) return rc;
  if (a.splits == 1) return HE_OK;
  const int rows = kJoinThreads / prompt_join_lanes(a.d);  // of a CTA
  const long long ctas = ((long long)a.batch * a.n_kv_heads * a.group * a.tokens + rows - 1) / rows;
  if (ctas > 0x7FFFFFFFLL) return fail(HE_ERR_UNSUPPORTED, "%d rows in one call", a.tokens);
  return launch_pdl(prompt_join_kernel, dim3((unsigned)ctas), kJoinThreads, 0, true, st, a);
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
  PromptArgs a{};
  a.tokens = a.keys = max_prompt_len, a.lens = a.kv_lens = prompt_len, a.doc_start = doc_start, a.prefix = prefix_len, a.splits = 1, a.self = 1;
  return attend_rows(a, cfg, mod, q, k, v, q_strides, kv_strides, out, out_strides, "max_prompt_len", nullptr, 0, static_cast<cudaStream_t>(stream));
}

size_t he_attend_cross_workspace_bytes(const he_config* cfg, int32_t max_q_len, int32_t max_kv_len) {
  if (check_config(cfg, true) || max_q_len < 1 || max_kv_len < 1 || max_q_len > kMaxTokens || max_kv_len > kMaxTokens) return 0;
  PromptArgs a{};
  a.batch = cfg->batch, a.n_kv_heads = cfg->n_kv_heads, a.group = cfg->group_size, a.d = cfg->head_dim, a.dtype = cfg->dtype, a.tokens = max_q_len, a.keys = max_kv_len;
  size_t most = 0;
  if (prompt_most_bytes(a, on_tensor_cores(a), &most)) return 0;
  return std::max(most, few_rows_workspace(cfg, std::min(max_q_len, kMaxGroup / cfg->group_size), 1));  // (of any number of keys the same)
}

int he_attend_cross(const he_config* cfg, const he_score_mod* mod, const void* q, const void* k, const void* v, const int64_t q_strides[3],
                    const int64_t kv_strides[3], const int32_t* q_len, int32_t max_q_len, const int32_t* kv_len, int32_t max_kv_len, const int32_t* q_pos,
                    const int32_t* first_key, const int32_t* prefix_len, void* out, const int64_t out_strides[3], void* workspace, size_t workspace_bytes,
                    void* stream) {
  PromptArgs a{};
  a.tokens = max_q_len, a.keys = max_kv_len, a.lens = q_len, a.kv_lens = kv_len, a.q_pos = q_pos, a.doc_start = first_key, a.prefix = prefix_len, a.splits = 1;
  a.all = q_pos == nullptr;
  if (q_pos == nullptr && (prefix_len != nullptr || (mod != nullptr && (mod->window != 0 || mod->slopes != nullptr))))
    return fail(HE_ERR_INVALID_ARG, "a window, slopes or a prefix without q_pos: rows without positions see every key");
  if (workspace != nullptr && !aligned16(workspace)) return fail(HE_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  return attend_rows(a, cfg, mod, q, k, v, q_strides, kv_strides, out, out_strides, "max_q_len", workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
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
