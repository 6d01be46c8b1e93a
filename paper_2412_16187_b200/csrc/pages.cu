// The cache of the full history, in pages: rows into it and back out (page_kernels.cuh), and a new token's attention over it (page_attend_kernels.cuh, and
// attend_kernels.cuh for what that does not take). Host side of these calls.
#include <cuda_runtime.h>

#include <cmath>

#include "attend_kernels.cuh"
#include "common.cuh"
#include "hashevict.h"
#include "few_rows.h"
#include "host_common.h"
#include "page_attend_kernels.cuh"
#include "page_kernels.cuh"

using namespace he;

int he::page_error_count() {
  int n = 0;
  return cudaMemcpyFromSymbol(&n, he::g_tc_error, sizeof(int)) == cudaSuccess ? n : -1;
}

namespace {

int check_pages(const he_config* cfg, const he_pages* p) {
  if (p == nullptr) return fail(HE_ERR_INVALID_ARG, "pages is null");
  if (!p->len || (p->max_pages != 0 && !p->page_table) || (p->n_pages != 0 && (!p->k_pages || !p->v_pages))) return fail(HE_ERR_INVALID_ARG, "pages has a null pointer");
  if (!aligned16(p->k_pages) || !aligned16(p->v_pages)) return fail(HE_ERR_INVALID_ARG, "pages must be 16-byte aligned");
  if (p->page_size < 16 || p->page_size > 128 || (p->page_size & (p->page_size - 1)) != 0)
    return fail(HE_ERR_INVALID_ARG, "page_size %d is not 16, 32, 64 or 128", p->page_size);
  if (p->n_pages < 0 || p->max_pages < 0) return fail(HE_ERR_INVALID_ARG, "n_pages %d / max_pages %d < 0", p->n_pages, p->max_pages);
  if ((long long)p->max_pages * p->page_size > kMaxTokens) return fail(HE_ERR_UNSUPPORTED, "%d pages of %d tokens in a sequence: more than 2^24 tokens", p->max_pages, p->page_size);
  if (p->eight_bit != 0 && p->eight_bit != 1) return fail(HE_ERR_INVALID_ARG, "eight_bit %d is not 0 or 1", p->eight_bit);
  if (p->eight_bit) {
    if (p->n_pages != 0 && (!p->k_scale || !p->v_scale)) return fail(HE_ERR_INVALID_ARG, "8-bit pages without scales");
    if (cfg->head_dim % 16 != 0) return fail(HE_ERR_UNSUPPORTED, "8-bit pages: head_dim %d is not a multiple of 16", cfg->head_dim);
  }
  return HE_OK;
}

template <int E, bool Q8>
int launch_append(const AppendArgs& a, const he_rotary& r, int v, dim3 grid, int threads, bool hold, cudaStream_t st) {
  constexpr int W = 16 / E;
  const size_t smem = hold ? append_smem(threads) : 0;
  auto as = [&](auto kernel) {
    if (int rc = set_smem(kernel, smem)) return rc;
    return launch_pdl(kernel, grid, threads, smem, true, st, a, r);
  };
  if (r.interleaved) return hold ? as(page_append_kernel<E, W, true, Q8, true>) : as(page_append_kernel<E, W, true, Q8, false>);
  if (v == W) return hold ? as(page_append_kernel<E, W, false, Q8, true>) : as(page_append_kernel<E, W, false, Q8, false>);
  return v == 4 ? as(page_append_kernel<E, 4, false, Q8, false>) : v == 2 ? as(page_append_kernel<E, 2, false, Q8, false>) : as(page_append_kernel<E, 1, false, Q8, false>);
}

// As many CTAs per unit as keep the grid within two per SM, at most 8 and no fewer than two tiles of tokens for each.
template <int E, int GP>
int launch_paged(const PagedAttendArgs& a, cudaStream_t st) {
  const long long units = (long long)a.cfg.batch * a.cfg.n_kv_heads;
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  int S = 1;
  while (S < 8 && 2 * S * units <= 2 * sms && 2 * S * 2 * kScoredSlots <= page_capacity(a.pages)) S *= 2;
  const int stages = E == 4 && S * units <= sms && scored_smem(S, 2, a.cfg.group_size, a.cfg.head_dim) <= kAttendMaxSmem ? 2 : 1;
  const size_t smem = scored_smem(S, stages, a.cfg.group_size, a.cfg.head_dim);
  auto kernel = attend_scored_kernel<E, GP, true>;
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
template <int E>
int launch_paged(const PagedAttendArgs& a, cudaStream_t st) {
  const int G = a.cfg.group_size;
  return G == 1 ? launch_paged<E, 1>(a, st) : G == 2 ? launch_paged<E, 2>(a, st) : G <= 4 ? launch_paged<E, 4>(a, st) : launch_paged<E, 8>(a, st);
}

// Tensor map of the rows of all pages of K or V: boxes of 64 bf16 channels, or of 64 or 128 codes, by a page's rows, at most 32. A map depends on the address and the
// shape alone, so the last few are kept per thread (a decode loop asks for the same ones at every token).
bool page_rows_tmap(const void* base, long long rows, int d, int box_rows, bool codes, CUtensorMap* out) {
  struct Entry {
    const void* base;
    long long rows;
    int d, box_rows, codes;
    CUtensorMap map;
  };
  constexpr int kEntries = 128;
  thread_local Entry known[kEntries] = {};
  Entry& e = known[(reinterpret_cast<uintptr_t>(base) >> 9) * 0x9E3779B97F4A7C15ull >> 57];
  if (e.base != base || e.rows != rows || e.d != d || e.box_rows != box_rows || e.codes != (int)codes) {
    const EncodeTiledFn encode = tmap_encoder();
    if (encode == nullptr || env_flag_set<5>("HE_DISABLE_TMA")) return false;
    const int wide = codes && d > 64;
    const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)d * (codes ? 1 : 2)};
    const cuuint32_t box[2] = {wide ? 128u : 64u, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    if (encode(&e.map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, codes && !wide ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
      e.base = nullptr;
      return false;
    }
    e.base = base, e.rows = rows, e.d = d, e.box_rows = box_rows, e.codes = codes;
  }
  *out = e.map;
  return true;
}

template <int D, bool Q8, int NBOX, bool LO, bool FOLD, bool ROWS = false>
int launch_page_attend(const TokenArgs& a, float* part, const PageMaps& maps, cudaStream_t st) {
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  auto kernel = page_attend_kernel<D, Q8, NBOX, LO, FOLD, ROWS>;
  static_assert(1024 + kPageRings<D, Q8> + kPageWarps<D, Q8> * (kMaxGroup * (D + 2)) * sizeof(float) <= 227 * 1024 - (Q8 ? 2048 : 1024), "rings and pieces beside what the kernel holds itself");
  const size_t smem = page_attend_smem<D, Q8>(a.cfg.group_size, a.cfg.head_dim);
  if (int rc = set_smem(kernel, smem)) return rc;
  if (int rc = launch_pdl(kernel, dim3((unsigned)sms), 32 * kPageWarps<D, Q8>, smem, true, st, a, part, maps)) return rc;
  if (sms == 1) return HE_OK;
  if (sms > kPageJoinThreads) return fail(HE_ERR_UNSUPPORTED, "%d multiprocessors", sms);
  return launch_pdl(page_join_kernel<ROWS>, dim3((unsigned)sms - 1), kPageJoinThreads, 0, true, st, a, part, sms);
}
template <int D>
int launch_page_attend(const TokenArgs& a, float* part, const PageMaps& maps, cudaStream_t st) {
  const bool two = a.pages.page_size < kPageGroup, fold = a.cfg.group_size <= 4;
  if (!a.pages.eight_bit)
    return two ? (fold ? launch_page_attend<D, false, 2, false, true>(a, part, maps, st) : launch_page_attend<D, false, 2, false, false>(a, part, maps, st))
               : (fold ? launch_page_attend<D, false, 1, false, true>(a, part, maps, st) : launch_page_attend<D, false, 1, false, false>(a, part, maps, st));
  if (a.cfg.dtype == HE_DTYPE_F32)
    return two ? (fold ? launch_page_attend<D, true, 2, true, true>(a, part, maps, st) : launch_page_attend<D, true, 2, true, false>(a, part, maps, st))
               : (fold ? launch_page_attend<D, true, 1, true, true>(a, part, maps, st) : launch_page_attend<D, true, 1, true, false>(a, part, maps, st));
  return two ? (fold ? launch_page_attend<D, true, 2, false, true>(a, part, maps, st) : launch_page_attend<D, true, 2, false, false>(a, part, maps, st))
             : (fold ? launch_page_attend<D, true, 1, false, true>(a, part, maps, st) : launch_page_attend<D, true, 1, false, false>(a, part, maps, st));
}

// Whether the tensor cores serve a call (where the driver makes tensor maps): rows of bf16 or of codes up to 128 channels, few enough for a map's coordinates.
bool page_tensor_cores(const he_config* cfg, const he_pages* p) {
  return p->n_pages > 0 && p->max_pages > 0 && (p->eight_bit || cfg->dtype == HE_DTYPE_BF16) && cfg->head_dim <= 128 && (long long)p->n_pages * cfg->n_kv_heads * p->page_size < 0x7FFFFF00LL &&
         page_line_fits(cfg, page_capacity(*p)) && getenv("HE_DISABLE_ATTEND_MMA") == nullptr;
}

// Tensor map of keys or values: {channel, token, head, sequence} in boxes of 64 channels x 32 tokens. An axis of one entry may come with any stride.
bool rows_over_tmap(const void* base, int d, int tokens, int heads, int batch, const int64_t* strides, CUtensorMap* out) {
  const EncodeTiledFn encode = tmap_encoder();
  if (encode == nullptr || env_flag_set<6>("HE_DISABLE_TMA")) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)tokens, (cuuint64_t)heads, (cuuint64_t)batch};
  cuuint64_t st[3] = {(cuuint64_t)strides[2] * 2, (cuuint64_t)strides[1] * 2, (cuuint64_t)strides[0] * 2};
  for (int i = 0; i < 3; ++i) {
    if (dims[i + 1] == 1) st[i] = (cuuint64_t)d * 2;
    if (st[i] == 0 || st[i] % 16 != 0 || st[i] >= (1ull << 40)) return false;
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)kPageGroup, 1, 1}, estr[4] = {1, 1, 1, 1};
  return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, st, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

size_t he::few_rows_workspace(const he_config* cfg, int rows, int keys) {
  int sms = 0;
  if (!few_rows(cfg, rows, keys) || sm_count(&sms)) return 0;
  return page_workspace(sms, rows * cfg->group_size, cfg->head_dim);
}

int he::launch_few_rows(const he_config* cfg, const RowsOverCall& c, cudaStream_t st) {
  TokenArgs a{};
  a.cfg = *cfg, a.cfg.group_size = cfg->group_size * c.rows, a.q = c.q;
  a.mod.scale_log2 = c.scale_log2, a.mod.cap_log2 = c.cap_log2, a.mod.inv_cap = c.inv_cap, a.mod.window = c.window, a.mod.slopes = c.slopes, a.mod.first_pos = c.first_key;
  a.pages.page_size = kPageGroup;
  a.over = {c.q_len, c.kv_len, c.q_pos, {c.q_strides[0], c.q_strides[1], c.q_strides[2]}, {c.out_strides[0], c.out_strides[1], c.out_strides[2]}, c.out, c.keys, c.rows};
  const int d = cfg->head_dim;
  PageMaps maps;
  if (!rows_over_tmap(c.k, d, c.keys, cfg->n_kv_heads, cfg->batch, c.kv_strides, &maps.k) || !rows_over_tmap(c.v, d, c.keys, cfg->n_kv_heads, cfg->batch, c.kv_strides, &maps.v))
    return -1;
  if (a.cfg.group_size <= 4)
    return d <= 64 ? launch_page_attend<64, false, 1, false, true, true>(a, c.part, maps, st) : launch_page_attend<128, false, 1, false, true, true>(a, c.part, maps, st);
  return d <= 64 ? launch_page_attend<64, false, 1, false, false, true>(a, c.part, maps, st) : launch_page_attend<128, false, 1, false, false, true>(a, c.part, maps, st);
}

extern "C" {

int he_page_append(const he_config* cfg, const he_pages* pages, const he_rotary* rotary, const void* k, const void* v, const int64_t kv_strides[3],
                   const int32_t* new_len, int32_t max_new, void* stream) {
  if (int rc = check_config(cfg, true)) return rc;
  if (int rc = check_pages(cfg, pages)) return rc;
  he_rotary none{};  // (halves of a row side by side in a warp write whole sectors: 512 MB of 8-bit pages 83 us, pieces next to each other 111)
  none.channels = cfg->head_dim % (2 * 16 / esize_of(cfg->dtype)) == 0 ? cfg->head_dim : 0;
  if (rotary != nullptr)
    if (int rc = check_rotary(rotary, cfg->head_dim)) return rc;
  if (max_new < 0) return fail(HE_ERR_INVALID_ARG, "max_new %d < 0", max_new);
  if (max_new == 0 || pages->max_pages == 0) return HE_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(HE_ERR_INVALID_ARG, "k or v is null or not 16-byte aligned");
  const int es = esize_of(cfg->dtype);
  if (int rc = check_strides("k / v", kv_strides, 3, es)) return rc;
  const he_rotary& r = rotary != nullptr ? *rotary : none;
  AppendArgs a{};
  a.pages = *pages, a.x[0] = k, a.x[1] = v, a.new_len = new_len, a.max_new = max_new, a.n_kv_heads = cfg->n_kv_heads, a.d = cfg->head_dim;
  for (int i = 0; i < 3; ++i) a.strides[i] = kv_strides[i];
  const int P = pages->page_size, V = rotary_piece(r, es);
  a.units = rotary_units(r, cfg->head_dim, V), a.turns = rotary != nullptr;
  const long long most = ((long long)max_new + P - 2) / P + 1;  // (they may begin on a page's last row)
  a.tiles = (int)(most < pages->max_pages ? most : pages->max_pages);
  const long long ctas = (long long)cfg->batch * a.tiles;
  if (ctas > 0x7FFFFFFFLL) return fail(HE_ERR_UNSUPPORTED, "%lld pages in one call", ctas);
  const int items = (max_new < P ? max_new : P) * a.units;  // of a page's new rows
  const bool hold = V == 16 / es && items <= kAppendThreads;
  const int threads = items < kAppendThreads ? (items + 31) / 32 * 32 : kAppendThreads;
  // Heads are shared out until there are enough CTAs for every SM, but a thread that has worked out its sines keeps at least four heads of a whole page. (16 prompts into pages of
  // 64 tokens: 44 us so, 51 with twice as many CTAs; of 128 tokens, an SM has one CTA at a time: 43 with two for each SM, 56 with four.)
  int sms = 0;
  if (int rc = sm_count(&sms)) return rc;
  const long long shares = ((threads > 512 ? 2LL : 4LL) * sms + ctas - 1) / ctas;
  a.heads_per_cta = (int)((cfg->n_kv_heads + shares - 1) / shares);
  const int least = max_new < P ? 1 : 4;
  if (a.heads_per_cta < least) a.heads_per_cta = least;
  if (a.heads_per_cta > cfg->n_kv_heads) a.heads_per_cta = cfg->n_kv_heads;
  const dim3 grid((unsigned)ctas, (unsigned)((cfg->n_kv_heads + a.heads_per_cta - 1) / a.heads_per_cta));
  if (grid.y > 65535) return fail(HE_ERR_UNSUPPORTED, "%d KV heads in one call", cfg->n_kv_heads);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (es == 2) return pages->eight_bit ? launch_append<2, true>(a, r, V, grid, threads, hold, st) : launch_append<2, false>(a, r, V, grid, threads, hold, st);
  return pages->eight_bit ? launch_append<4, true>(a, r, V, grid, threads, hold, st) : launch_append<4, false>(a, r, V, grid, threads, hold, st);
}

int he_page_read(const he_config* cfg, const he_pages* pages, const int32_t* first, int32_t max_rows, void* k_out, void* v_out, const int64_t kv_strides[3],
                 void* stream) {
  if (int rc = check_config(cfg, true)) return rc;
  if (int rc = check_pages(cfg, pages)) return rc;
  if (max_rows < 0) return fail(HE_ERR_INVALID_ARG, "max_rows %d < 0", max_rows);
  if (max_rows == 0 || pages->max_pages == 0) return HE_OK;
  if (!k_out && !v_out) return fail(HE_ERR_INVALID_ARG, "neither k_out nor v_out is given");
  if (!aligned16(k_out) || !aligned16(v_out)) return fail(HE_ERR_INVALID_ARG, "k_out or v_out is not 16-byte aligned");
  if (k_out == v_out) return fail(HE_ERR_INVALID_ARG, "k_out and v_out overlap");
  const int es = esize_of(cfg->dtype);
  if (int rc = check_strides("k_out / v_out", kv_strides, 3, es)) return rc;
  const long long sizes[3] = {cfg->batch, cfg->n_kv_heads, max_rows};
  if (int rc = check_apart("k_out / v_out", kv_strides, sizes, 3, cfg->head_dim)) return rc;
  if (cfg->batch > 65535) return fail(HE_ERR_UNSUPPORTED, "batch %d > 65535 in one call", cfg->batch);
  ReadArgs a{};
  a.pages = *pages, a.out[0] = k_out, a.out[1] = v_out, a.first = first, a.max_rows = max_rows, a.n_kv_heads = cfg->n_kv_heads, a.d = cfg->head_dim;
  for (int i = 0; i < 3; ++i) a.strides[i] = kv_strides[i];
  a.sides = k_out && v_out ? 2 : 1, a.side = k_out ? 0 : 1;
  const long long most = (long long)max_rows < page_capacity(*pages) ? max_rows : page_capacity(*pages), ctas = (most + kReadRows - 2) / kReadRows + 1;
  const int chunks = cfg->head_dim * es / 16;  // of a row
  const long long heads = (long long)a.sides * cfg->n_kv_heads;
  if (heads > 65535) return fail(HE_ERR_UNSUPPORTED, "%d KV heads in one call", cfg->n_kv_heads);
  const dim3 grid((unsigned)ctas, (unsigned)heads, (unsigned)cfg->batch), block((unsigned)chunks, (unsigned)(kReadThreads / chunks));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto as = [&](auto kernel) { return launch_pdl(kernel, grid, block, 0, true, st, a); };
  if (es == 2) return pages->eight_bit ? as(page_read_kernel<2, true>) : as(page_read_kernel<2, false>);
  return pages->eight_bit ? as(page_read_kernel<4, true>) : as(page_read_kernel<4, false>);
}

size_t he_page_attend_workspace_bytes(const he_config* cfg, const he_pages* pages) {
  int sms = 0;
  if (check_config(cfg, true) || check_pages(cfg, pages) || !page_tensor_cores(cfg, pages) || sm_count(&sms)) return 0;
  return page_workspace(sms, cfg->group_size, cfg->head_dim);
}

int he_page_attend(const he_config* cfg, const he_pages* pages, const he_score_mod* mod, const void* q, const int32_t* first_pos, float* out, void* workspace,
                   size_t workspace_bytes, void* stream) {
  if (int rc = check_config(cfg, true)) return rc;
  if (int rc = check_pages(cfg, pages)) return rc;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return fail(HE_ERR_INVALID_ARG, "q or out is null or not 16-byte aligned");
  if (cfg->batch > 65535) return fail(HE_ERR_UNSUPPORTED, "batch %d > 65535 in one call", cfg->batch);
  TokenArgs a{};
  a.cfg = *cfg, a.pages = *pages, a.q = q, a.out = out;
  if (pages->n_pages == 0) a.pages.k_pages = a.pages.v_pages = const_cast<void*>(q);  // (copies of no bytes are given an address all the same)
  if (int rc = check_mod(mod, cfg->head_dim, &a.mod.scale_log2, &a.mod.cap_log2, &a.mod.inv_cap, &a.mod.window, &a.mod.slopes)) return rc;
  a.mod.first_pos = first_pos;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (workspace != nullptr && !aligned16(workspace)) return fail(HE_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  if (page_tensor_cores(cfg, pages)) {
    const size_t need = he_page_attend_workspace_bytes(cfg, pages);
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return fail(HE_ERR_WORKSPACE, "workspace of %zu bytes, %zu are needed", workspace_bytes, need);
    const long long rows = (long long)pages->n_pages * cfg->n_kv_heads * pages->page_size;
    const int box = pages->page_size < kPageGroup ? pages->page_size : kPageGroup;
    PageMaps maps;
    if (page_rows_tmap(pages->k_pages, rows, cfg->head_dim, box, pages->eight_bit, &maps.k) && page_rows_tmap(pages->v_pages, rows, cfg->head_dim, box, pages->eight_bit, &maps.v))
      return cfg->head_dim <= 64 ? launch_page_attend<64>(a, static_cast<float*>(workspace), maps, st) : launch_page_attend<128>(a, static_cast<float*>(workspace), maps, st);
  }
  return pages->eight_bit ? launch_paged<1>(a, st) : cfg->dtype == HE_DTYPE_BF16 ? launch_paged<2>(a, st) : launch_paged<4>(a, st);
}

}  // extern "C"
