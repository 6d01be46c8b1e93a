// he_attend_prompt: attention of prompts over themselves, out_i = sum_j softmax_j(x_ij) V_j with
//   x_ij = cap(scale q_i . k_j) - slope |i - j|   for the j of one interval [lo_i, hi_i) per token (document, window, past, prefix).
// One interval per row means that a tile of rows walks over one run of key tiles and compares column numbers only in those at the run's ends.
// All kernels keep the running maximum, the sum of the weights and the unnormalised output of a row in fp32, in log2 units.
//
//   prompt_tc_kernel      bf16, head sizes up to 128: two tiles of 128 rows x 128 keys at a time on the tensor cores (tcgen05).
//   prompt_fp32_kernel    any dtype and head size: 64 rows x 64 keys at a time on the CUDA cores.
//
// Values in hidden places. Hidden keys get a weight of zero by selection, whatever their score is; a hidden V row that holds an infinity or a
// NaN would still turn the product 0 * V into NaN. V rows behind the prompt's end are therefore read as zeros, and a
// row whose output has come out as NaN is computed once more over its visible keys alone (prompt_row_again), which costs nothing where it does not happen.
#pragma once
#include <cuda_bf16.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace he {

struct PromptArgs {
  const void *q, *k, *v;
  void* out;
  long long qs[3], ks[3], os[3];  // element strides (sequence, head, token) of q, of k and v, of out
  int batch, n_kv_heads, group, d, dtype, tokens;
  const int32_t* lens;       // [B]
  const int32_t* doc_start;  // [B, tokens] or null
  const int32_t* prefix;     // [B] or null
  const float* slopes;       // [Hkv*G] or null
  float scale_log2, cap_log2, inv_cap;  // scores in log2 units: scale_log2 * q.k, or cap_log2 * tanh(inv_cap * q.k)
  int window;
};

constexpr float kPromptLog2e = 1.4426950408889634f;

// The keys that token i sees; empty for i >= n.
__device__ __forceinline__ void prompt_interval(const PromptArgs& a, int s, int i, int n, int& lo, int& hi) {
  lo = 0, hi = 0;
  if (i >= n) return;
  if (a.window > 0) lo = max(lo, i - a.window + 1);
  if (a.doc_start != nullptr) lo = max(lo, a.doc_start[(long long)s * a.tokens + i]);
  hi = i + 1;
  if (a.prefix != nullptr) hi = max(hi, a.prefix[s]);
  hi = min(hi, n);
}

__device__ __forceinline__ float prompt_element(const void* p, long long at, int dtype) {
  return dtype == HE_DTYPE_BF16 ? bf16_bits_to_f32(static_cast<const uint16_t*>(p)[at]) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void prompt_store(void* p, long long at, int dtype, float f) {
  if (dtype == HE_DTYPE_BF16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(f);
  else static_cast<float*>(p)[at] = f;
}

// One row by one warp, over its visible keys alone.
static __device__ __noinline__ void prompt_row_again(const PromptArgs& a, int s, int head, int i, int n) {
  const int lane = threadIdx.x & 31, kv = head / a.group;
  int lo, hi;
  prompt_interval(a, s, i, n, lo, hi);
  const long long q0 = s * a.qs[0] + head * a.qs[1] + i * a.qs[2], k0 = s * a.ks[0] + kv * a.ks[1];
  const float slope = a.slopes != nullptr ? a.slopes[head] * kPromptLog2e : 0.f;
  float q[kMaxDim / 32], o[kMaxDim / 32], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int c = 0; c < kMaxDim / 32; ++c) q[c] = lane + 32 * c < a.d ? prompt_element(a.q, q0 + lane + 32 * c, a.dtype) : 0.f, o[c] = 0.f;
  for (int j = lo; j < hi; ++j) {
    float dot = 0.f;
#pragma unroll
    for (int c = 0; c < kMaxDim / 32; ++c)
      if (lane + 32 * c < a.d) dot = fmaf(q[c], prompt_element(a.k, k0 + j * a.ks[2] + lane + 32 * c, a.dtype), dot);
    for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, off);
    float x = a.cap_log2 > 0.f ? a.cap_log2 * tanhf(dot * a.inv_cap) : dot * a.scale_log2;
    x -= slope * (float)abs(i - j);
    const float mx = fmaxf(m, x), mn = mx == -INFINITY ? 0.f : mx, corr = exp2f(m - mn), p = exp2f(x - mn);
    l = l * corr + p;
    m = mx;
#pragma unroll
    for (int c = 0; c < kMaxDim / 32; ++c)
      if (lane + 32 * c < a.d) o[c] = o[c] * corr + p * prompt_element(a.v, k0 + j * a.ks[2] + lane + 32 * c, a.dtype);
  }
  const long long o0 = s * a.os[0] + head * a.os[1] + i * a.os[2];
#pragma unroll
  for (int c = 0; c < kMaxDim / 32; ++c)
    if (lane + 32 * c < a.d) prompt_store(a.out, o0 + lane + 32 * c, a.dtype, l != 0.f ? o[c] / l : 0.f);
}

// ------------------------------------------------------------------------------------------------ CUDA cores
//
// 64 rows of one query head per CTA, 64 keys at a time. Thread (ty, tx) of 16 x 16 holds the scores of rows 4 ty .. + 3 and keys
// 4 tx .. + 3, and of the output the same rows and channels 4 tx .. + 3 of every 64. Q and K lie in shared memory channel by channel, so that
// both are read as four values at a time; the weights go through shared memory key by key.
constexpr int kPromptRows = 64, kPromptThreads = 256, kPromptPitch = 68;
inline size_t prompt_fp32_smem(int d) { return sizeof(float) * (2 * (size_t)d * kPromptPitch + 64 * (size_t)d + 64 * (size_t)kPromptPitch); }

template <int NQ>  // groups of 64 channels
__global__ void __launch_bounds__(kPromptThreads) prompt_fp32_kernel(const PromptArgs a, const int tiles) {
  extern __shared__ __align__(16) float psm_[];
  const int d = a.d, tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 31;
  const int heads = a.n_kv_heads * a.group;
  const int head = blockIdx.x % heads, s = (blockIdx.x / heads) % a.batch, tile = tiles - 1 - blockIdx.x / heads / a.batch;
  const int kv = head / a.group, i0 = tile * kPromptRows;
  float* qt = psm_;                   // [d][68]
  float* kt = qt + d * kPromptPitch;  // [d][68]
  float* vs = kt + d * kPromptPitch;  // [64][d]
  float* pt = vs + 64 * d;            // [64 keys][68]
  __shared__ int run[2];
  griddep_launch_dependents();
  griddep_wait();
  const int n = min(max(a.lens[s], 0), a.tokens);
  if (i0 >= n) return;
  if (tid == 0) run[0] = 0x7FFFFFFF, run[1] = 0;
  int lo[4], hi[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) prompt_interval(a, s, i0 + 4 * ty + r, n, lo[r], hi[r]);
  __syncthreads();
  if (tx == 0)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (lo[r] < hi[r]) atomicMin(&run[0], lo[r]), atomicMax(&run[1], hi[r]);
  const long long q0 = s * a.qs[0] + head * a.qs[1], k0 = s * a.ks[0] + kv * a.ks[1];
  for (int idx = tid; idx < 64 * d; idx += kPromptThreads) {
    const int r = idx / d, c = idx % d;
    qt[c * kPromptPitch + r] = i0 + r < n ? prompt_element(a.q, q0 + (i0 + r) * a.qs[2] + c, a.dtype) : 0.f;
  }
  const float slope = a.slopes != nullptr ? a.slopes[head] * kPromptLog2e : 0.f;
  float m[4], l[4], o[4][4 * NQ];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * NQ; ++c) o[r][c] = 0.f;
  }
  __syncthreads();
  const int j_begin = run[0] / 64 * 64, j_end = run[1];
  for (int j0 = j_begin; j0 < j_end; j0 += 64) {
    __syncthreads();  // the last tile has been read
    for (int idx = tid; idx < 64 * d; idx += kPromptThreads) {
      const int r = idx / d, c = idx % d, j = j0 + r;
      kt[c * kPromptPitch + r] = j < n ? prompt_element(a.k, k0 + j * a.ks[2] + c, a.dtype) : 0.f;
      vs[idx] = j < n ? prompt_element(a.v, k0 + j * a.ks[2] + c, a.dtype) : 0.f;
    }
    __syncthreads();
    float x[4][4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[r][e] = 0.f;
    for (int c = 0; c < d; ++c) {
      const float4 q4 = *reinterpret_cast<const float4*>(qt + c * kPromptPitch + 4 * ty), k4 = *reinterpret_cast<const float4*>(kt + c * kPromptPitch + 4 * tx);
      const float qv[4] = {q4.x, q4.y, q4.z, q4.w}, kv4[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[r][e] = fmaf(qv[r], kv4[e], x[r][e]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = i0 + 4 * ty + r;
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = j0 + 4 * tx + e;
        float y = a.cap_log2 > 0.f ? a.cap_log2 * tanhf(x[r][e] * a.inv_cap) : x[r][e] * a.scale_log2;
        y -= slope * (float)abs(i - j);
        x[r][e] = j >= lo[r] && j < hi[r] ? y : -INFINITY;
        top = fmaxf(top, x[r][e]);
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
      const float mx = fmaxf(m[r], top), mn = mx == -INFINITY ? 0.f : mx, corr = exp2f(m[r] - mn);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[r][e] = exp2f(x[r][e] - mn), sum += x[r][e];
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
      l[r] = l[r] * corr + sum;
      m[r] = mx;
#pragma unroll
      for (int c = 0; c < 4 * NQ; ++c) o[r][c] *= corr;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<float4*>(pt + (4 * tx + e) * kPromptPitch + 4 * ty) = make_float4(x[0][e], x[1][e], x[2][e], x[3][e]);
    __syncwarp();  // rows 4 ty .. + 3 are written and read by the same half warp
    for (int j = 0; j < 64; ++j) {
      const float4 p4 = *reinterpret_cast<const float4*>(pt + j * kPromptPitch + 4 * ty);
      const float pv[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int c = 64 * q + 4 * tx;
        if (c < d) {
          const float4 v4 = *reinterpret_cast<const float4*>(vs + j * d + c);
          const float vv[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][4 * q + e] = fmaf(pv[r], vv[e], o[r][4 * q + e]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = i0 + 4 * ty + r;
    const long long o0 = s * a.os[0] + head * a.os[1] + i * a.os[2];
    bool bad = false;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 64 * q + 4 * tx + e;
        const float f = l[r] != 0.f ? o[r][4 * q + e] / l[r] : 0.f;
        if (i < n && c < d) prompt_store(a.out, o0 + c, a.dtype, f), bad |= f != f;
      }
    const uint32_t again = __ballot_sync(0xFFFFFFFFu, bad);
    __syncwarp();
#pragma unroll
    for (int w = 0; w < 2; ++w)  // the rows of this warp's two ty
      if ((again >> (16 * w)) & 0xFFFFu) prompt_row_again(a, s, head, i0 + 4 * ((tid - lane) / 16 + w) + r, n);
  }
}

// ------------------------------------------------------------------------------------------------ tensor cores
//
// A CTA works on two tiles of 128 rows that walk over the same blocks of 128 keys: two query heads of one KV head (the same tokens) where the
// group is even, else 256 tokens of one head. Per block and tile S = Q K^T (128 x 128, fp32 in tensor memory), the softmax's weights P, and
// O += P V (128 x D, fp32 in tensor memory) with P read from tensor memory, where it takes the place of S. While one tile's softmax runs, the
// tensor cores work for the other tile.
//
//   warps 0-3, 4-7   softmax of tile 0, of tile 1: a thread owns a row, so that its maximum and sum need no exchange. The output is rescaled
//                    only when a row's maximum has grown by more than 2^8 since the last time (weights up to 256 lose nothing in fp32 or bf16).
//   warp 8           issues the products: S of the next block of a tile right behind O += P V of this one
//   warp 9           copies Q, then K and V block by block through a ring of TMA tiles (128-byte swizzle)
//
// Registers: 384 threads are launched with 168 each (64,512); warps 0-7 take 208, warps 8-11 keep 80: 256 * 208 + 128 * 80 = 63,488.
// Channels from d up to D are filled with zeros by the tensor maps.
constexpr int kPtThreads = 384, kPtTile = 128, kPtMmaWarp = 8, kPtLoadWarp = 9;
constexpr int kPtSoftRegs = 208, kPtOtherRegs = 80;
constexpr float kPtSlack = 8.f;  // log2 of how far weights may exceed 1 before the output is rescaled

template <int D>
struct PromptTc {
  static constexpr int kTileBytes = kPtTile * D * 2;
  static constexpr int kStages = D == 128 ? 4 : 8;  // K or V tiles in flight
  static constexpr size_t kSmem = 1024 + (size_t)(2 + kStages) * kTileBytes;
};

struct PromptMaps {
  alignas(64) CUtensorMap q, k, v;
};

__device__ __forceinline__ void pt_mma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
// 32 columns of this thread's tensor-memory lane
__device__ __forceinline__ void pt_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
      "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]),
      "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]),
      "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void pt_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float pt_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float pt_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pt_pack(float x, float y) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}

// Shared-memory matrix descriptor of V as the B operand: rows are the products' K index, channels contiguous (MN-major), 128-byte
// swizzle: 8-row groups 1024 bytes apart, groups of 64 channels a box (128 rows) apart.
__device__ __forceinline__ uint64_t pt_desc_mn128(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((kPtTile * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kPtThreads, 1) prompt_tc_kernel(const PromptArgs a, const int tiles, const int by_heads, const __grid_constant__ PromptMaps maps) {
  using T = PromptTc<D>;
  constexpr int NS = T::kStages, NH = D / 64, BOX = kPtTile * 128;
  extern __shared__ __align__(16) unsigned char pt_smem_raw[];
  __shared__ __align__(8) unsigned long long full_s[NS], empty_s[NS], qfull_s[2], sfull_s[2], pfull_s[2], odone_s[2], drain_s;
  __shared__ int run_s[2][4];  // per tile: first key seen, end of the keys seen, first and end of the keys that all rows see
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  griddep_launch_dependents();
  griddep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int heads = a.n_kv_heads * a.group, per = by_heads ? heads / 2 : heads;
  const int p_idx = blockIdx.x % per, s = (blockIdx.x / per) % a.batch, tile = tiles - 1 - (int)(blockIdx.x / per / a.batch);
  const int n = min(max(a.lens[s], 0), a.tokens);
  const int tok0 = by_heads ? tile * kPtTile : tile * 2 * kPtTile;
  if (tok0 >= n) return;
  auto head_of = [&](int t) { return by_heads ? 2 * p_idx + t : p_idx; };
  auto tok_of = [&](int t) { return by_heads ? tok0 : tok0 + t * kPtTile; };
  const uint32_t smem0 = (smem_u32(pt_smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = smem0, ring = smem0 + 2 * T::kTileBytes;
  volatile int* abort_flag = &abort_s;

  if (tid == 0) {
#pragma unroll
    for (int i = 0; i < NS; ++i) mbar_init(smem_u32(&full_s[i]), 1), mbar_init(smem_u32(&empty_s[i]), 1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&qfull_s[t]), 1), mbar_init(smem_u32(&sfull_s[t]), 1), mbar_init(smem_u32(&odone_s[t]), 1);
      mbar_init(smem_u32(&pfull_s[t]), kPtTile);
      run_s[t][0] = 0x7FFFFFFF, run_s[t][1] = 0, run_s[t][2] = 0, run_s[t][3] = 0x7FFFFFFF;
    }
    mbar_init(smem_u32(&drain_s), 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kPtMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  __syncthreads();
  int lo = 0, hi = 0;
  if (warp < 8) {
    const int t = warp >> 2, i = tok_of(t) + (tid & (kPtTile - 1));
    prompt_interval(a, s, i, n, lo, hi);
    const bool some = lo < hi;
    const int first = __reduce_min_sync(0xFFFFFFFFu, some ? lo : 0x7FFFFFFF), end = __reduce_max_sync(0xFFFFFFFFu, some ? hi : 0);
    const int all_lo = __reduce_max_sync(0xFFFFFFFFu, i >= n ? 0 : some ? lo : 0x7FFFFFFF), all_hi = __reduce_min_sync(0xFFFFFFFFu, i >= n ? 0x7FFFFFFF : hi);
    if (lane == 0) atomicMin(&run_s[t][0], first), atomicMax(&run_s[t][1], end), atomicMax(&run_s[t][2], all_lo), atomicMin(&run_s[t][3], all_hi);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  // blocks of keys [begin, end) of each tile and of both
  int jb[2], je[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const bool some = run_s[t][1] > 0;
    jb[t] = some ? run_s[t][0] / kPtTile : 0, je[t] = some ? (run_s[t][1] + kPtTile - 1) / kPtTile : 0;
  }
  const int j_begin = jb[0] == je[0] ? jb[1] : jb[1] == je[1] ? jb[0] : min(jb[0], jb[1]), j_end = max(je[0], je[1]);

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax and output of tile t
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPtSoftRegs));
    const int t = warp >> 2, row = tid & (kPtTile - 1), i = tok_of(t) + row, head = head_of(t);
    const uint32_t lane_base = tmem + ((uint32_t)(warp & 3) << 21);  // this warp's 32 lanes
    const uint32_t s_t = lane_base + t * kPtTile, o_t = lane_base + 2 * kPtTile + t * D;
    const int all_lo = run_s[t][2], all_hi = run_s[t][3];
    const float slope = BIAS ? a.slopes[head] * kPromptLog2e : 0.f;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    const int steps = je[t] - jb[t];
    for (int it = 0; it < steps; ++it) {
      const int j0 = (jb[t] + it) * kPtTile;
      ok = mbar_wait_warp(smem_u32(&sfull_s[t]), it & 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      uint32_t raw[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tc_ld32(s_t + 32 * c, raw[c]);
      tc_wait_ld();
      float x[128];
#pragma unroll
      for (int c = 0; c < 128; ++c) x[c] = __uint_as_float(raw[c >> 5][c & 31]);
      if (CAP) {
        const float two = a.inv_cap * (2.f * kPromptLog2e), top = a.cap_log2;
#pragma unroll
        for (int c = 0; c < 128; ++c) x[c] = fmaf(-2.f * top, pt_rcp(pt_ex2(x[c] * two) + 1.f), top);  // tanh z = 1 - 2 / (e^2z + 1)
      }
      if (BIAS) {
        const float away = (float)(j0 - i);
#pragma unroll
        for (int c = 0; c < 128; ++c) {
          const float y = CAP ? x[c] : x[c] * a.scale_log2;
          x[c] = fmaf(-slope, fabsf(away + (float)c), y);
        }
      }
      if (j0 < all_lo || j0 + kPtTile > all_hi) {
        const uint32_t from = (uint32_t)(lo - j0), span = (uint32_t)(hi - lo);
        const bool some = lo < hi;
#pragma unroll
        for (int c = 0; c < 128; ++c) x[c] = some && (uint32_t)c - from < span ? x[c] : -INFINITY;
      }
      float top = fmaxf(x[0], x[1]);
#pragma unroll
      for (int c = 2; c < 128; c += 2) top = fmaxf(top, fmaxf(x[c], x[c + 1]));
      const float scale = CAP || BIAS ? 1.f : a.scale_log2;
      const float mx = fmaxf(m, top * scale);
      if (__any_sync(0xFFFFFFFFu, mx > m + kPtSlack)) {  // (m = -inf: the first keys that a row sees)
        const float corr = mx == -INFINITY ? 1.f : pt_ex2(m - mx);
        m = mx;
        l *= corr;
        if (it > 0) {  // the product of the block before is done: S of this one was issued behind it
#pragma unroll
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            tc_ld32(o_t + c, o);
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr);
            pt_st32(o_t + c, o);
          }
        }
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      uint32_t w[2][32];
#pragma unroll
      for (int c = 0; c < 128; c += 2) {
        const float p0 = pt_ex2(fmaf(x[c], scale, -ref)), p1 = pt_ex2(fmaf(x[c + 1], scale, -ref));
        sum[(c >> 1) & 3] += p0 + p1;
        w[c >> 6][(c >> 1) & 31] = pt_pack(p0, p1);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      pt_st32(s_t, w[0]);
      pt_st32(s_t + 32, w[1]);
      pt_wait_st();
      tc_fence_before();
      mbar_arrive(smem_u32(&pfull_s[t]));
    }
    if (ok && steps > 0) ok = mbar_wait_warp(smem_u32(&odone_s[t]), 0, abort_flag);
    if (ok) {
      tc_fence_after();
      const float inv = l != 0.f ? 1.f / l : 0.f;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + (s * a.os[0] + head * a.os[1] + i * a.os[2]);
      bool bad = false;
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        if (steps > 0) {
          tc_ld32(o_t + c, o);
          tc_wait_ld();
        }
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          float f[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            f[u] = steps > 0 && inv != 0.f ? __uint_as_float(o[e + u]) * inv : 0.f;
            bad |= c + e < a.d && f[u] != f[u];
          }
          if (i < n && c + e < a.d)
            *reinterpret_cast<uint4*>(out + c + e) = make_uint4(pt_pack(f[0], f[1]), pt_pack(f[2], f[3]), pt_pack(f[4], f[5]), pt_pack(f[6], f[7]));
        }
      }
      uint32_t again = __ballot_sync(0xFFFFFFFFu, bad && i < n);
      __syncwarp();
      for (; again != 0u; again &= again - 1u) prompt_row_again(a, s, head, i - lane + __ffs(again) - 1, n);
    }
    tc_fence_before();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPtOtherRegs));
    if (warp == kPtLoadWarp) {
      // ---------------------------------------------------------------- copies
      int slot = 0, used = 0;  // ring place of the next tile, tiles asked for so far
      if (lane == 0) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (je[t] > jb[t]) {
            const uint32_t bar = smem_u32(&qfull_s[t]);
            mbar_arrive_expect_tx(bar, T::kTileBytes);
#pragma unroll
            for (int h = 0; h < NH; ++h) tma_load_4d(q_smem + t * T::kTileBytes + h * BOX, &maps.q, 64 * h, tok_of(t), head_of(t), s, bar);
          }
      }
      const int kv = head_of(0) / a.group;
      for (int item = 0; item < 2 * (j_end - j_begin); ++item) {
        if (used >= NS && !mbar_wait_warp(smem_u32(&empty_s[slot]), ((used / NS) - 1) & 1, abort_flag)) break;
        if (lane == 0) {
          const uint32_t bar = smem_u32(&full_s[slot]);
          mbar_arrive_expect_tx(bar, T::kTileBytes);
#pragma unroll
          for (int h = 0; h < NH; ++h)
            tma_load_4d(ring + slot * T::kTileBytes + h * BOX, (item & 1) ? &maps.v : &maps.k, 64 * h, (j_begin + (item >> 1)) * kPtTile, kv, s, bar);
        }
        ++used;
        slot = slot + 1 == NS ? 0 : slot + 1;
      }
      __syncwarp();
      if (__any_sync(0xFFFFFFFFu, *abort_flag != 0)) {  // let what is in flight land before shared memory is given up
        for (int t = 0; t < 2; ++t)
          if (je[t] > jb[t]) mbar_drain(smem_u32(&qfull_s[t]), 0);
        for (int u = max(0, used - NS); u < used; ++u) mbar_drain(smem_u32(&full_s[u % NS]), (u / NS) & 1);
      }
    } else if (warp == kPtMmaWarp) {
      // ---------------------------------------------------------------- products (issued by one elected lane)
      constexpr uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((kPtTile / 8) << 17) | ((kPtTile / 16) << 24);
      constexpr uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) /* B is MN-major */ | ((D / 8) << 17) | ((kPtTile / 16) << 24);
      bool ok = true;
      auto slot_of = [&](int item) { return item % NS; };
      auto landed = [&](int item) { ok = ok && mbar_wait_warp(smem_u32(&full_s[slot_of(item)]), (item / NS) & 1, abort_flag); };
      auto qk = [&](int t, int item) {
        if (!ok) return;
        const uint64_t ad = umma_desc_k128(q_smem + t * T::kTileBytes), bd = umma_desc_k128(ring + slot_of(item) * T::kTileBytes);
        if (tc_elect()) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint64_t at = (uint64_t)(((ks >> 2) * BOX + (ks & 3) * 32) >> 4);
            tc_mma_bf16(tmem + t * kPtTile, ad + at, bd + at, idesc_qk, ks != 0);
          }
          tc_commit(smem_u32(&sfull_s[t]));
        }
        __syncwarp();
      };
      auto pv = [&](int t, int item, int it, bool last) {
        ok = ok && mbar_wait_warp(smem_u32(&pfull_s[t]), it & 1, abort_flag);
        if (!ok) return;
        tc_fence_after();
        const uint64_t bd = pt_desc_mn128(ring + slot_of(item) * T::kTileBytes);
        if (tc_elect()) {
#pragma unroll
          for (int ks = 0; ks < kPtTile / 16; ++ks)
            pt_mma_ts(tmem + 2 * kPtTile + t * D, tmem + t * kPtTile + 8 * ks, bd + (uint64_t)((ks * 16 * 128) >> 4), idesc_pv, it > 0 || ks != 0);
          if (last) tc_commit(smem_u32(&odone_s[t]));
        }
        __syncwarp();
      };
      auto release = [&](int item) {
        if (ok && tc_elect()) tc_commit(smem_u32(&empty_s[slot_of(item)]));
        __syncwarp();
      };
      auto active = [&](int t, int j) { return j >= jb[t] && j < je[t]; };
      for (int j = j_begin - 1; j < j_end && ok; ++j) {
        // O += P V of block j, S of block j + 1, tile by tile
        const int item = 2 * (j - j_begin);  // block j's K; its V is the next, block j + 1's K the one after
        if (j >= j_begin) {
          landed(item + 1);
          const int rows = n - j * kPtTile;
          if (ok && rows < kPtTile) {  // V rows behind the prompt's end hold anything: zeros
            for (int u = lane; u < (kPtTile - rows) * 8 * NH; u += 32) {
              const int h = u / ((kPtTile - rows) * 8), at = u % ((kPtTile - rows) * 8);
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring + slot_of(item + 1) * T::kTileBytes + h * BOX + rows * 128 + at * 16), "r"(0) : "memory");
            }
            fence_proxy_async();
            __syncwarp();
          }
        }
        if (j + 1 < j_end) landed(item + 2);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (j >= j_begin && active(t, j)) pv(t, item + 1, j - jb[t], j + 1 == je[t]);
          if (j + 1 < j_end && active(t, j + 1)) {
            if (j + 1 == jb[t]) ok = ok && mbar_wait_warp(smem_u32(&qfull_s[t]), 0, abort_flag);
            qk(t, item + 2);
          }
        }
        if (j >= j_begin) release(item + 1);
        if (j + 1 < j_end) release(item + 2);
      }
      const bool gave_up = __any_sync(0xFFFFFFFFu, *abort_flag != 0);
      if (gave_up) {  // products in flight end before tensor memory is given up
        if (tc_elect()) tc_commit(smem_u32(&drain_s));
        __syncwarp();
        mbar_drain(smem_u32(&drain_s), 0);
      }
    }
    __syncwarp();
  }
  __syncthreads();
  if (tid == 0 && abort_s) atomicAdd(&g_tc_error, 1);
  if (warp == kPtMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

}  // namespace he
