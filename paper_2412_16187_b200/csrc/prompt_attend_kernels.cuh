// he_attend_prompt: attention of prompts over themselves, out_i = sum_j softmax_j(x_ij) V_j with
//   x_ij = cap(scale q_i . k_j) - slope |i - j|   for the j of one interval [lo_i, hi_i) per token (document, window, past, prefix).
// One interval per row means that a tile of rows walks over one run of key tiles and compares column numbers only in those at the run's ends.
// All kernels keep the running maximum, the sum of the weights and the unnormalised output of a row in fp32, in log2 units.
//
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

}  // namespace he
