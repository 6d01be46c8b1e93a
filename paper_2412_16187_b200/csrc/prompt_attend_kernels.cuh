// he_attend_prompt: attention of prompts over themselves, out_i = sum_j softmax_j(x_ij) V_j with
//   x_ij = cap(scale q_i . k_j) - slope |i - j|   for the j of one interval [lo_i, hi_i) per token (document, window, past, prefix).
// One interval per row means that a tile of rows walks over one run of key tiles and compares column numbers only in those at the run's ends.
// All kernels keep the running maximum, the sum of the weights and the unnormalised output of a row in fp32, in log2 units.
//
//   prompt_tc_kernel      bf16, head sizes up to 128: two tiles of 128 rows x 128 keys at a time on the tensor cores (tcgen05).
//   prompt_fp32_kernel    any dtype and head size: 64 or 16 rows x 64 keys at a time on the CUDA cores.
//
// Values in hidden places. Hidden keys get a weight of zero by selection, whatever their score is; a hidden V row that holds an infinity or a
// NaN would still turn the product 0 * V into NaN. V rows behind the prompt's end are therefore read as zeros, and a row whose output has come
// out as NaN is computed once more over its visible keys alone where what it hides can be the reason (prompt_rows_again). It cannot where the sum of the
// weights is a NaN (a score that the row sees), where no V row that its tile has multiplied by zero holds anything but numbers, or where
// V rows that it sees are NaN in the same channels. Looking costs a warp one run over the rows in question for its 32 rows of output.
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
  float near_end;  // kPtNearEnd where the near form of the tanh can be written for inv_cap, else -1
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

__device__ __forceinline__ void prompt_store(void* p, long long at, int dtype, float f) {
  if (dtype == HE_DTYPE_BF16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(f);
  else static_cast<float*>(p)[at] = f;
}

// Elements of a 16-byte chunk as fp32: eight, or four.
template <int ES>
__device__ __forceinline__ void prompt_unpack(const uint4& chunk, float (&f)[16 / ES]) {
  const uint32_t w[4] = {chunk.x, chunk.y, chunk.z, chunk.w};
#pragma unroll
  for (int e = 0; e < 16 / ES; ++e) f[e] = ES == 4 ? __uint_as_float(w[e % 4]) : __uint_as_float((e & 1) ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
}

// Up to four rows of a head, row[0] <= row[1] <= ..., by one warp, each over its visible keys alone: 32 keys at a time, a lane for the scores of each, then for
// the channels of one chunk (of 1 / per of the keys where a row has fewer chunks than there are lanes). `beat`: raised now and then for those
// who wait meanwhile. Four rows over 2048 keys at d = 128 take 0.6 ms.
constexpr int kPromptAgain = 4;
template <int ES>
static __device__ __noinline__ void prompt_compute_again(const PromptArgs& a, int s, int head, const int (&row)[kPromptAgain], int n, volatile int* beat) {
  constexpr int EPC = 16 / ES, SLOTS = ES == 4 ? 2 : 1, RB = kPromptAgain;  // elements of a chunk; chunks of a lane (rows have up to 64)
  const uint32_t all_lanes = 0xFFFFFFFFu;
  const int lane = threadIdx.x & 31, kv = head / a.group, cpr = a.d / EPC;
  const int per = cpr < 32 ? 32 / cpr : 1, sub = cpr < 32 ? lane / cpr : 0, c = cpr < 32 ? lane % cpr : lane;
  auto chunk = [&](const void* p, long long at_row, int at) { return *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + at_row * ES + 16 * at); };
  const long long q0 = s * a.qs[0] + head * a.qs[1], k0 = s * a.ks[0] + kv * a.ks[1];
  const float slope = a.slopes != nullptr ? a.slopes[head] * kPromptLog2e : 0.f;
  int lo[RB], hi[RB], begin = 0x7FFFFFFF, end = 0;
  float m[RB], l[RB], o[RB][SLOTS][EPC];  // l: of this lane's keys; o: of this lane's chunks and keys
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    prompt_interval(a, s, row[b], n, lo[b], hi[b]);
    begin = min(begin, lo[b]), end = max(end, hi[b]);
    m[b] = -INFINITY, l[b] = 0.f;
#pragma unroll
    for (int w = 0; w < SLOTS; ++w)
#pragma unroll
      for (int e = 0; e < EPC; ++e) o[b][w][e] = 0.f;
  }
  for (int j0 = begin; j0 < end; j0 += 32) {
    if (beat != nullptr && ((j0 - begin) & 1023) == 0 && lane == 0) *beat = *beat + 1;
    const int j = min(j0 + lane, end - 1), count = min(end - j0, 32);
    float dot[RB] = {};
#pragma unroll 4
    for (int at = 0; at < cpr; ++at) {
      float kf[EPC];
      prompt_unpack<ES>(chunk(a.k, k0 + j * a.ks[2], at), kf);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        float qf[EPC];
        prompt_unpack<ES>(chunk(a.q, q0 + row[b] * a.qs[2], at), qf);
#pragma unroll
        for (int e = 0; e < EPC; ++e) dot[b] = fmaf(qf[e], kf[e], dot[b]);
      }
    }
    float p[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      float x = a.cap_log2 > 0.f ? a.cap_log2 * tanhf(dot[b] * a.inv_cap) : dot[b] * a.scale_log2;
      x -= slope * (float)abs(row[b] - j);
      x = j0 + lane >= lo[b] && j0 + lane < hi[b] ? x : -INFINITY;
      float mx = fmaxf(m[b], x);
      for (int off = 16; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(all_lanes, mx, off));
      const float mn = mx == -INFINITY ? 0.f : mx, corr = exp2f(m[b] - mn);
      p[b] = exp2f(x - mn);
      l[b] = l[b] * corr + p[b];
      m[b] = mx;
#pragma unroll
      for (int w = 0; w < SLOTS; ++w)
#pragma unroll
        for (int e = 0; e < EPC; ++e) o[b][w][e] *= corr;
    }
#pragma unroll 4
    for (int t = 0; t < count; t += per) {
      const int key = j0 + t + sub;
      float pj[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) pj[b] = __shfl_sync(all_lanes, p[b], (t + sub) & 31);
      if (sub < per && t + sub < count)
#pragma unroll
        for (int w = 0; w < SLOTS; ++w)
          if (c + 32 * w < cpr) {
            float vf[EPC];
            prompt_unpack<ES>(chunk(a.v, k0 + key * a.ks[2], c + 32 * w), vf);
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
              for (int e = 0; e < EPC; ++e) o[b][w][e] = fmaf(pj[b], key >= lo[b] && key < hi[b] ? vf[e] : 0.f, o[b][w][e]);
          }
    }
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    for (int off = 16; off > 0; off >>= 1) l[b] += __shfl_xor_sync(all_lanes, l[b], off);
    const long long o0 = s * a.os[0] + head * a.os[1] + row[b] * a.os[2];
#pragma unroll
    for (int w = 0; w < SLOTS; ++w)
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        float sum = o[b][w][e];
        for (int k = 1; k < per; ++k) sum += __shfl_sync(all_lanes, o[b][w][e], (c + k * cpr) & 31);  // (per > 1: cpr < 32)
        if (sub == 0 && c + 32 * w < cpr) prompt_store(a.out, o0 + EPC * (c + 32 * w) + e, a.dtype, l[b] != 0.f ? sum / l[b] : 0.f);
      }
  }
}

// A bit for each element of 16 bytes that is a NaN or, without `nan_only`, an infinity.
__device__ __forceinline__ uint32_t prompt_odd_bits(const uint4& chunk, int dtype, bool nan_only) {
  const uint32_t w[4] = {chunk.x, chunk.y, chunk.z, chunk.w}, least = nan_only ? 1u : 0u;
  uint32_t bits = 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (dtype == HE_DTYPE_BF16)
      bits |= (uint32_t)((w[e] & 0x7FFFu) >= 0x7F80u + least) << (2 * e) | (uint32_t)((w[e] >> 16 & 0x7FFFu) >= 0x7F80u + least) << (2 * e + 1);
    else
      bits |= (uint32_t)((w[e] & 0x7FFFFFFFu) >= 0x7F800000u + least) << e;
  return bits;
}

// The rows i0 + b of one head, b a bit of `again`, whose outputs are stored, hold a NaN and have a number for the sum of their weights; their tile has
// multiplied the V rows [from, to). Computes those anew whose NaNs may come from rows that they hide. By a whole warp.
static __device__ __noinline__ void prompt_rows_again(const PromptArgs& a, int s, int head, int i0, uint32_t again, int n, int from, int to, volatile int* beat = nullptr) {
  constexpr int STEPS = 4;  // loads in flight
  const uint32_t all_lanes = 0xFFFFFFFFu;
  const int lane = threadIdx.x & 31, kv = head / a.group, es = esize_of(a.dtype), cpr = a.d * es / 16;  // (16-byte chunks of a row: up to 64)
  const int per = cpr < 32 ? 32 / cpr : 1, sub = cpr < 32 ? lane / cpr : 0, c = cpr < 32 ? lane % cpr : lane;  // rows at a time; this lane's row of them and chunk
  const char* v = static_cast<const char*>(a.v) + (s * a.ks[0] + kv * a.ks[1]) * es;
  const char* out = static_cast<const char*>(a.out) + (s * a.os[0] + head * a.os[1]) * es;
  auto odd = [&](const char* p, long long stride, int row, int chunk, bool nan_only) -> uint32_t {
    return chunk < cpr ? prompt_odd_bits(*reinterpret_cast<const uint4*>(p + row * stride * es + 16 * chunk), a.dtype, nan_only) : 0u;
  };
  auto hides_odd = [&](int row) { return (odd(v, a.ks[2], row, c, false) | odd(v, a.ks[2], row, c + 32, false)) != 0u; };
  auto alive = [&](int step) {
    if (beat != nullptr && (step & 63) == 0 && lane == 0) *beat = *beat + 1;
  };
  int lo, hi;
  prompt_interval(a, s, i0 + lane, n, lo, hi);
  bool mine = (again >> lane) & 1u;
  // The last row behind what they see, and the first before it, that is not all numbers.
  const int begin = __reduce_min_sync(all_lanes, mine ? hi : to), end = __reduce_max_sync(all_lanes, mine ? lo : from);
  int last = -1, first = 0x7FFFFFFF, step = 0;
  for (int j = to; j > begin && last < 0; j -= STEPS * per) {
    int found = -1;
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int row = j - 1 - u * per - sub;
      if (sub < per && row >= begin && hides_odd(row)) found = max(found, row);
    }
    last = __reduce_max_sync(all_lanes, found);
    alive(++step);
  }
  for (int j = from; j < end && first == 0x7FFFFFFF; j += STEPS * per) {
    int found = 0x7FFFFFFF;
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int row = j + u * per + sub;
      if (sub < per && row < end && hides_odd(row)) found = min(found, row);
    }
    first = __reduce_min_sync(all_lanes, found);
    alive(++step);
  }
  mine = mine && (last >= hi || first < lo);
  again = __ballot_sync(all_lanes, mine);
  if (again == 0u) return;
  // Channels that are NaN in rows that all the others see too, from the last on until they explain every output.
  const int seen_begin = __reduce_max_sync(all_lanes, mine ? lo : 0), seen_end = __reduce_min_sync(all_lanes, mine ? hi : 0x7FFFFFFF);
  uint32_t want[2] = {0u, 0u}, have[2] = {0u, 0u}, known[2] = {0u, 0u};
  for (uint32_t rest = again; rest != 0u; rest &= rest - 1u)
#pragma unroll
    for (int w = 0; w < 2; ++w) want[w] |= odd(out, a.os[2], i0 + __ffs(rest) - 1, c + 32 * w, true);
  for (int j = seen_end; j > seen_begin; j -= STEPS * per) {
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int row = j - 1 - u * per - sub;
      if (sub < per && row >= seen_begin)
#pragma unroll
        for (int w = 0; w < 2; ++w) have[w] |= odd(v, a.ks[2], row, c + 32 * w, true);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      known[w] = have[w];
      for (int k = 0; k < per && cpr < 32; ++k) known[w] |= __shfl_sync(all_lanes, have[w], c + k * cpr);
    }
    if (__all_sync(all_lanes, ((want[0] & ~known[0]) | (want[1] & ~known[1])) == 0u)) break;
    alive(++step);
  }
  int row[kPromptAgain], rows = 0;
  for (uint32_t rest = again; rest != 0u;) {
    const int i = i0 + __ffs(rest) - 1;
    rest &= rest - 1u;
    const uint32_t open = (odd(out, a.os[2], i, c, true) & ~known[0]) | (odd(out, a.os[2], i, c + 32, true) & ~known[1]);
    if (__any_sync(all_lanes, open != 0u)) {
#pragma unroll
      for (int b = 0; b < kPromptAgain; ++b)
        if (b >= rows) row[b] = i;  // (places that stay empty repeat the last row)
      ++rows;
    }
    if (rows == kPromptAgain || (rest == 0u && rows > 0)) {
      if (es == 2) prompt_compute_again<2>(a, s, head, row, n, beat);
      else prompt_compute_again<4>(a, s, head, row, n, beat);
      rows = 0;
    }
  }
}

// ------------------------------------------------------------------------------------------------ CUDA cores
//
// 16 R rows of one query head per CTA, 64 keys at a time. Thread (ty, tx) of 16 x 16 holds the scores of rows R ty .. + R - 1 and keys
// tx, tx + 16, tx + 32, tx + 48, and of the output the same rows and channels 4 tx .. + 3 of every 64. Q and K lie in shared memory row by row, four
// floats longer than the row, so that the 16 threads that read neighbouring keys meet every bank once; the weights go through shared memory key by key, in the place of K.
// What bounds it: issue slots (69 % used), which the products share with the loads that feed them (R = 4: 8 of 16 bytes for 64 products; shared memory is 61 %
// busy) and with the softmax; the FMA pipe is 50 % busy, waiting for copies or at barriers 5 % of the stalls. 4 x 32 heads of 2048 tokens at d = 128 take
// 4.5 ms: 31 TFLOP/s, of about 70 that the FMA pipe has. With one CTA an SM instead of two it was
// 6.0 ms there, and 32 heads of 2048 tokens at d = 64 took 1.03 ms beside 0.70. bf16 heads of 136 to 256, which come here too: 23 TFLOP/s (16 heads of 2048
// tokens at d = 256 1.5 ms).
// R = 1 for calls that would leave SMs idle: 5 x 311 tokens of one head at d = 128 take 35 us beside 76 with R = 4 (44 without a tile ahead);
// 32 heads of 1024 tokens, which fill the SMs, 319 us with R = 4 beside 772.
constexpr int kPromptThreads = 256;
template <int R>
constexpr int kPromptPitch = 16 * R + 4;  // of the weights
template <int R>
inline size_t prompt_fp32_smem(int d, int stages) {
  const size_t keys = 64 * (size_t)(d + 4), weights = 64 * (size_t)kPromptPitch<R>;  // the weights take the place of the K tile
  return sizeof(float) * ((size_t)16 * R * (d + 4) + (size_t)stages * ((keys > weights ? keys : weights) + 64 * (size_t)d));
}
// 16 bytes into shared memory, or zeros
__device__ __forceinline__ void prompt_copy16(void* smem_dst, const void* gmem_src, bool some) {
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(smem_dst);
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(gmem_src), "r"(some ? 16u : 0u) : "memory");
}

// fp32 rows are copied asynchronously, with `stages` = 2 a tile of keys ahead (calls that leave an SM to one CTA).
template <int NQ, int R>  // groups of 64 channels, rows of a thread
__global__ void __launch_bounds__(kPromptThreads, NQ <= 2 ? 2 : 1) prompt_fp32_kernel(const __grid_constant__ PromptArgs a, const int tiles, const int stages) {
  extern __shared__ __align__(16) float psm_[];
  constexpr int PP = kPromptPitch<R>;
  constexpr int UNROLL = R == 1 ? 8 : 2;  // one row has few loads in flight otherwise
  const int d = a.d, pitch = d + 4, tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 31;
  const int heads = a.n_kv_heads * a.group;
  const int head = blockIdx.x % heads, s = (blockIdx.x / heads) % a.batch, tile = tiles - 1 - blockIdx.x / heads / a.batch;
  const int kv = head / a.group, i0 = tile * 16 * R;
  float* qs = psm_;                // [16 R][d + 4]
  float* ks = qs + 16 * R * pitch; // [64][d + 4]
  const int keys_floats = 64 * max(pitch, PP), stage_floats = keys_floats + 64 * d;  // K tile (then the weights [64 keys][16 R + 4]), V tile [64][d]
  __shared__ int run[2];
  griddep_launch_dependents();
  griddep_wait();
  const int n = min(max(a.lens[s], 0), a.tokens);
  if (i0 >= n) return;
  if (tid == 0) run[0] = 0x7FFFFFFF, run[1] = 0;
  int lo[R], hi[R];
#pragma unroll
  for (int r = 0; r < R; ++r) prompt_interval(a, s, i0 + R * ty + r, n, lo[r], hi[r]);
  __syncthreads();
  if (tx == 0)
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (lo[r] < hi[r]) atomicMin(&run[0], lo[r]), atomicMax(&run[1], hi[r]);
  const long long q0 = s * a.qs[0] + head * a.qs[1], k0 = s * a.ks[0] + kv * a.ks[1];
  const int es = esize_of(a.dtype), cpr = d * es / 16;  // 16-byte chunks of a row
  auto chunk = [&](const void* p, long long row_at, int c) {
    return __ldg(reinterpret_cast<const uint4*>(static_cast<const char*>(p) + row_at * es) + c);
  };
  for (int idx = tid; idx < 16 * R * cpr; idx += kPromptThreads) {
    const int r = idx / cpr, c = idx % cpr;
    store_chunk(qs + r * pitch, i0 + r < n ? chunk(a.q, q0 + (i0 + r) * a.qs[2], c) : make_uint4(0u, 0u, 0u, 0u), c, a.dtype);
  }
  const float slope = a.slopes != nullptr ? a.slopes[head] * kPromptLog2e : 0.f;
  float m[R], l[R], o[R][4 * NQ];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * NQ; ++c) o[r][c] = 0.f;
  }
  __syncthreads();
  const int j_begin = run[0], j_end = run[1];  // (nothing ahead of the first key that a row sees is read)
  const int r_first = tid / cpr, c_first = tid % cpr, r_step = kPromptThreads / cpr, c_step = kPromptThreads % cpr;
  const bool async = a.dtype == HE_DTYPE_F32;
  auto fetch = [&](int j0, int stage) {
    float* kt = ks + stage * stage_floats;
    float* vt = kt + keys_floats;
#pragma unroll 4
    for (int r = r_first, c = c_first; r < 64;) {
      const int j = j0 + r;
      const long long at = k0 + (j < n ? j : 0) * a.ks[2];
      if (async) {
        prompt_copy16(kt + r * pitch + 4 * c, static_cast<const float*>(a.k) + at + 4 * c, j < n);
        prompt_copy16(vt + r * d + 4 * c, static_cast<const float*>(a.v) + at + 4 * c, j < n);
      } else {
        uint4 k4 = make_uint4(0u, 0u, 0u, 0u), v4 = k4;
        if (j < n) k4 = chunk(a.k, at, c), v4 = chunk(a.v, at, c);
        store_chunk(kt + r * pitch, k4, c, HE_DTYPE_BF16);
        store_chunk(vt + r * d, v4, c, HE_DTYPE_BF16);
      }
      r += r_step, c += c_step;
      if (c >= cpr) c -= cpr, ++r;
    }
    cp_async_commit();
  };
  if (stages == 2 && j_begin < j_end) fetch(j_begin, 0);
  for (int j0 = j_begin, stage = 0; j0 < j_end; j0 += 64, stage ^= stages - 1) {
    if (stages == 2) {
      if (j0 + 64 < j_end) {
        fetch(j0 + 64, stage ^ 1);
        cp_async_wait_pending(1);
      } else {
        cp_async_wait_all();
      }
    } else {
      fetch(j0, 0);
      cp_async_wait_all();
    }
    __syncthreads();
    const float* kt = ks + stage * stage_floats;
    const float* vt = kt + keys_floats;
    float* pt = ks + stage * stage_floats;
    float x[R][4];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[r][e] = 0.f;
#pragma unroll UNROLL
    for (int c = 0; c < d; c += 4) {
      float4 q4[R], k4[4];
#pragma unroll
      for (int r = 0; r < R; ++r) q4[r] = *reinterpret_cast<const float4*>(qs + (R * ty + r) * pitch + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) k4[e] = *reinterpret_cast<const float4*>(kt + (tx + 16 * e) * pitch + c);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[r][e] = fmaf(q4[r].w, k4[e].w, fmaf(q4[r].z, k4[e].z, fmaf(q4[r].y, k4[e].y, fmaf(q4[r].x, k4[e].x, x[r][e]))));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = i0 + R * ty + r;
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = j0 + tx + 16 * e;
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
    __syncthreads();  // K has been read
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (R == 4) *reinterpret_cast<float4*>(pt + (tx + 16 * e) * PP + 4 * ty) = make_float4(x[0][e], x[1][e], x[2][e], x[3][e]);
      else pt[(tx + 16 * e) * PP + ty] = x[0][e];
    }
    __syncwarp();  // a row's weights are written and read by the same half warp
#pragma unroll UNROLL
    for (int j = 0; j < 64; ++j) {
      __align__(16) float pv[R];
      if constexpr (R == 4) *reinterpret_cast<float4*>(pv) = *reinterpret_cast<const float4*>(pt + j * PP + 4 * ty);
      else pv[0] = pt[j * PP + ty];
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int c = 64 * q + 4 * tx;
        if (c < d) {
          const float4 v4 = *reinterpret_cast<const float4*>(vt + j * d + c);
          const float vv[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][4 * q + e] = fmaf(pv[r], vv[e], o[r][4 * q + e]);
        }
      }
    }
    __syncthreads();  // the tile has been read
  }
  uint32_t again = 0u;  // rows of this warp with a NaN that a score does not explain
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int i = i0 + R * ty + r;
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
    const uint32_t odd = __ballot_sync(0xFFFFFFFFu, bad && l[r] == l[r]);
#pragma unroll
    for (int w = 0; w < 2; ++w)  // the rows of this warp's two ty
      if ((odd >> (16 * w)) & 0xFFFFu) again |= 1u << (R * w + r);
  }
  __syncwarp();
  if (again != 0u) prompt_rows_again(a, s, head, i0 + R * (tid - lane) / 16, again, n, j_begin, min(j_begin + (j_end - j_begin + 63) / 64 * 64, n));
}

// ------------------------------------------------------------------------------------------------ tensor cores
//
// A work item is two tiles of 128 rows that walk over the same blocks of 128 keys, the last first (a bias by distance then lets the
// running maximum stand, and no output is rescaled): two query heads of one KV head (the same tokens) where the
// group is even, else 256 tokens of one head. Per block and tile S = Q K^T (128 x 128, fp32 in tensor memory), the softmax's weights P, and
// O += P V (128 x D, fp32 in tensor memory) with P read from tensor memory, where it takes the place of S. While one tile's softmax runs, the
// tensor cores work for the other tile.
//
//   warps 0-3, 4-7   softmax of tile 0, of tile 1: a thread owns a row, so that its maximum and sum need no exchange. The output is rescaled
//                    only when a row's maximum has grown by more than 2^8 since the last time (weights up to 256 lose nothing in fp32 or bf16).
//   warp 8           issues the products: S of the next block of a tile right behind O += P V of this one
//   warp 9           copies Q, then K and V block by block through a ring of TMA tiles (128-byte swizzle)
//   warp 10          fetches work: one CTA per SM is resident, takes over the grid's waiting CTAs one after another (cluster launch control)
//                    and works out which blocks each needs while the others are busy with the item before
//
// The items come with the prompts' last tokens first, as those see the most keys. The roles run on from item to item: the next one's Q, K
// and first S are under way while the rows of this one are written.
//
// Registers: 384 threads are launched with 168 each, 64,512 in all; warps 0-7 take 224, warps 8-11 keep 56: 256 * 224 + 128 * 56 = 64,512. The compiler
// allocates for 168 and spills in every instance (12 to 56 bytes of stores a thread without a cap, 100 to 156 with one).
// Channels from d up to D are filled with zeros by the tensor maps.
constexpr int kPtThreads = 384, kPtTile = 128, kPtMmaWarp = 8, kPtLoadWarp = 9, kPtWorkWarp = 10;
constexpr int kPtSoftRegs = 224, kPtOtherRegs = 56;
constexpr int kPtAsk = 4;           // steps of an item that are still to be asked for when the next item is fetched
constexpr int kPtReaders = 10;       // warps that read an item: softmax, products, copies
constexpr float kPtSlack = 8.f;      // log2 of how far weights may exceed 1 before the output is rescaled
constexpr float kPtTanhEnd = 7.f;    // see pt_tanh
constexpr float kPtNearEnd = 0.7f;   // see pt_tanh_near
constexpr float kPtNearInv = 1e-5f, kPtNearMost = 1e5f;  // the powers of a smaller or larger factor leave fp32: PromptArgs::near_end is -1 there

template <int D>
struct PromptTc {
  static constexpr int kTileBytes = kPtTile * D * 2;
  static constexpr int kStages = D == 128 ? 2 : 4;  // places of the ring: K of a block and V of the block before
  static constexpr size_t kSmem = 1024 + (size_t)(2 + 2 * kStages) * kTileBytes;
};

struct PromptMaps {
  alignas(64) CUtensorMap q, k, v;
};

// An item: its rows, the first key that any of them sees (block j holds the keys base + 128 j on: what lies before, say the padding ahead of a prompt, is
// never multiplied), how many keys of the last block lie within the prompt, and per tile the blocks of keys [jb, je) that it needs and at
// which steps from the last of them on, [all_from, all_to), its rows see every key of the block.
struct PtItem {
  int some, s, n, p, tok0, base, last_rows;
  int jb[2], je[2], all_from[2], all_to[2];
};

// One product or commit, issued by the lane of a converged warp that has `leader` set: a predicate on the instruction, so that descriptors stay in
// uniform registers.
__device__ __forceinline__ void pt_mma_ss(uint32_t leader, uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void pt_mma_ts(uint32_t leader, uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void pt_commit(uint32_t leader, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader)
      : "memory");
}
// 16 columns of this thread's tensor-memory lane
__device__ __forceinline__ void pt_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
      "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void pt_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
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
// Maximum and minimum that hand a NaN on.
__device__ __forceinline__ float pt_max(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float pt_max3(float x, float y, float z) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
__device__ __forceinline__ float pt_max3_abs(float x, float y, float z) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
__device__ __forceinline__ float pt_min(float x, float y) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
// Pairs of fp32 values, two to an instruction.
struct pt2 {
  unsigned long long v;
  __device__ __forceinline__ pt2() {}
  __device__ __forceinline__ pt2(float x, float y) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y)); }
  __device__ __forceinline__ void get(float& x, float& y) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
};
__device__ __forceinline__ pt2 pt_fma(pt2 a, pt2 b, pt2 c) {
  pt2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ pt2 pt_mul(pt2 a, pt2 b) {
  pt2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ pt2 pt_add(pt2 a, pt2 b) {
  pt2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

// 2^x of N pairs on the FMA pipe, for x <= 100; below -125 it is 2^-125. x = k + f with k the nearest integer, 2^f on [-1/2, 1/2] by the cubic
// with the least largest relative error (7.5e-5, fitted by reweighted least squares), k added to the exponent. The weights are then rounded to bf16 (up to
// 3.9e-3), and their sum is taken of the same values. The pairs go through it side by side: one alone is a chain of ten dependent steps.
template <int N>
__device__ __forceinline__ void pt_ex2_fma(const pt2* x, float* y) {
  const pt2 magic(12582912.f, 12582912.f), back(-12582912.f, -12582912.f), minus(-1.f, -1.f);
  pt2 k[N], f[N], r[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float a, b;
    x[i].get(a, b);
    f[i] = pt2(pt_max(a, -125.f), pt_max(b, -125.f));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) k[i] = pt_add(f[i], magic);  // the low bits hold the integer
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = pt_add(k[i], back);
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = pt_fma(r[i], minus, f[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = pt_fma(f[i], pt2(0.05517166480422020f, 0.05517166480422020f), pt2(0.2426111400127411f, 0.2426111400127411f));
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = pt_fma(r[i], f[i], pt2(0.6932609677314758f, 0.6932609677314758f));
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = pt_fma(r[i], f[i], pt2(0.9999280571937561f, 0.9999280571937561f));
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float r0, r1, k0, k1;
    r[i].get(r0, r1), k[i].get(k0, k1);
    y[2 * i] = __int_as_float(__float_as_int(r0) + (__float_as_int(k0) << 23));
    y[2 * i + 1] = __int_as_float(__float_as_int(r1) + (__float_as_int(k1) << 23));
  }
}

// tanh(inv x) / inv of N pairs, |inv x| <= 0.7: x P(x^2), the cubic P(inv^2 x^2) with the least largest relative error (6.7e-6, fitted by reweighted
// least squares) and the powers of inv in its coefficients.
struct PtNear {
  float c0, c1, c2, c3;
};
__device__ __forceinline__ PtNear pt_near(float inv) {
  const float i2 = inv * inv;
  return {0.9999933242797852f, -0.33289045095443726f * i2, 0.12864211201667786f * i2 * i2, -0.03729049488902092f * i2 * i2 * i2};
}
template <int N>
__device__ __forceinline__ void pt_tanh_near(pt2* x, const PtNear& c) {
  pt2 w[N], r[N];
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = pt_mul(x[i], x[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = pt_fma(w[i], pt2(c.c3, c.c3), pt2(c.c2, c.c2));
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = pt_fma(r[i], w[i], pt2(c.c1, c.c1));
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = pt_fma(r[i], w[i], pt2(c.c0, c.c0));
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = pt_mul(r[i], x[i]);
}

// tanh of N pairs, any z: z N(z^2) / D(z^2) with cubics N and D, both 1 at 0, fitted for the least largest error on [-7, 7] (1.4e-6, relative for |z| < 1), where
// tanh 7 = 1 - 1.7e-6 stands for all beyond. One reciprocal serves a pair: D is at most 91. (By exponentials it takes two special-function
// operations an element, beside the softmax's own one the pipe that bounds the kernel.)
template <int N>
__device__ __forceinline__ void pt_tanh(pt2* z) {
  const pt2 one(1.f, 1.f);
  pt2 w[N], nu[N], de[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float a, b;
    z[i].get(a, b);
    z[i] = pt2(pt_min(pt_max(a, -kPtTanhEnd), kPtTanhEnd), pt_min(pt_max(b, -kPtTanhEnd), kPtTanhEnd));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {  // a NaN goes on in the numerator alone: the reciprocal is shared with a neighbour that may be seen where this one is hidden
    float a, b;
    pt_mul(z[i], z[i]).get(a, b);
    w[i] = pt2(fminf(a, kPtTanhEnd * kPtTanhEnd), fminf(b, kPtTanhEnd * kPtTanhEnd));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) de[i] = pt_fma(w[i], pt2(0.00014415701319693802f, 0.00014415701319693802f), pt2(0.02116040722518346f, 0.02116040722518346f));
#pragma unroll
  for (int i = 0; i < N; ++i) nu[i] = pt_fma(w[i], pt2(4.0026867816318985e-06f, 4.0026867816318985e-06f), pt2(0.0022948283489213545f, 0.0022948283489213545f));
#pragma unroll
  for (int i = 0; i < N; ++i) de[i] = pt_fma(de[i], w[i], pt2(0.4565702597687332f, 0.4565702597687332f));
#pragma unroll
  for (int i = 0; i < N; ++i) nu[i] = pt_fma(nu[i], w[i], pt2(0.1232431128784306f, 0.1232431128784306f));
#pragma unroll
  for (int i = 0; i < N; ++i) de[i] = pt_fma(de[i], w[i], one);
#pragma unroll
  for (int i = 0; i < N; ++i) nu[i] = pt_fma(nu[i], w[i], one);
#pragma unroll
  for (int i = 0; i < N; ++i) nu[i] = pt_mul(nu[i], z[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float d0, d1;
    de[i].get(d0, d1);
    const float r = pt_rcp(d0 * d1);
    z[i] = pt_mul(nu[i], pt_mul(pt2(r, r), pt2(d1, d0)));
  }
}

// Shared-memory matrix descriptor of V as the B operand: rows are the products' K index, channels contiguous (MN-major), 128-byte
// swizzle: 8-row groups 1024 bytes apart, groups of 64 channels a box (128 rows) apart.
__device__ __forceinline__ uint64_t pt_desc_mn128(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((kPtTile * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// Bounded wait of a whole warp on another role's work, which may take as long as a row of the longest prompt: the limit counts from the last
// sign of life (`beat`, raised by the softmax warps every few blocks) on.
__device__ __forceinline__ bool pt_wait_on(uint32_t bar, uint32_t parity, volatile int* abort_flag, volatile int* beat) {
  bool got = false;
#pragma unroll 1
  for (int seen = *beat;;) {
#pragma unroll 1
    for (uint32_t i = 0; i < kTcSpinLimit && !got; ++i) {
      got = mbar_try_wait(bar, parity);
      if (*abort_flag) break;
    }
    if (got || *abort_flag) break;
    const int now = *beat;
    if (now == seen) {
      *abort_flag = 1;
      break;
    }
    seen = now;
  }
  return __all_sync(0xFFFFFFFFu, got);
}
__device__ __forceinline__ bool pt_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, volatile int* beat) {
  if (__builtin_expect(__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity)), 1)) return true;
  return pt_wait_on(bar, parity, abort_flag, beat);
}

// The same for the roles beside the softmax, what follows the first poll in one place (for each kernel, next to its code: one place for all costs up to 2 %).
template <int D, bool CAP, bool BIAS>
static __device__ __noinline__ bool pt_wait_far(uint32_t bar, uint32_t parity, volatile int* abort_flag, volatile int* beat) {
  return pt_wait_on(bar, parity, abort_flag, beat);
}
template <int D, bool CAP, bool BIAS>
__device__ __forceinline__ bool pt_wait_small(uint32_t bar, uint32_t parity, volatile int* abort_flag, volatile int* beat) {
  if (__builtin_expect(__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity)), 1)) return true;
  return pt_wait_far<D, CAP, BIAS>(bar, parity, abort_flag, beat);
}

// The grid's next waiting CTA, cancelled and taken over: asked for by one lane, answered in 16 bytes of shared memory.
__device__ __forceinline__ void pt_ask_work(uint32_t answer, uint32_t bar) {
  fence_proxy_async();
  mbar_arrive_expect_tx(bar, 16u);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
__device__ __forceinline__ bool pt_read_work(uint32_t answer, int& cta) {
  uint32_t some, x;
  asm volatile(
      "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t"
      "ld.shared.b128 r, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "mov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
      : "=r"(some), "=r"(x)
      : "r"(answer)
      : "memory");
  cta = (int)x;
  return some != 0;
}

// EMU of a row's 64 pairs of weights are computed on the FMA pipe: the special-function pipe (16 a cycle and SM) takes 2048 cycles for a block's
// 2 x 128 x 128 weights, as long as the block's products at D = 128 and twice as long at D = 64. With hardly any there (EMU = 1), 16 heads of 8192 tokens
// took 324 us instead of 316 with a cap, 128 heads of 512 tokens 33 instead of 31; with cap and slopes together the FMA pipe is the
// busier one (d = 64: 322 us with EMU = 2, 347 with 8).
//
// What bounds it (16 heads of 8192 tokens, d = 128: 231 us = 1.19 PFLOP/s plain, 311 with a cap, 267 with slopes, 358 with both; d = 64: 190, 285, 220, 321; with
// scores beyond 0.7 of the cap, whose blocks go through both forms of the tanh, 688 and 645): a tile's way around, some 3500 cycles for a block. Its softmax takes about 2000 of them, as one thread walks over a row of 128 in the registers it
// has; then the products P V and the next S take 1024 of their own and 400 of hand-overs, while the other tile's softmax runs. The
// issue slots are 36 to 40 % used, the special-function pipe 40 %, the tensor pipe 50 %. An item adds about 9000 cycles (first S, last product, output).
// Short prompts have few blocks an item and are bound by that (32 heads of 1024 tokens: 24 us).
// At D = 64 a quarter of tensor memory (columns 384 to 511) is not used: P lies where S was, and the next S of a tile waits for it.
// Tried and slower: blocks of 64 keys with two places for S (0.90 PFLOP/s), one warp that polls both tiles for whichever is ready (0.81), weights handed over
// in two or four parts, 208 / 80 registers (more spills in the softmax).
template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kPtThreads, 1) prompt_tc_kernel(const __grid_constant__ PromptArgs a, const int tiles, const int by_heads,
                                                                   const __grid_constant__ PromptMaps maps) {
  using T = PromptTc<D>;
  constexpr int NS = T::kStages, NH = D / 64, BOX = kPtTile * 128, EMU = CAP && BIAS ? 2 : CAP || BIAS ? 8 : 12;
  extern __shared__ __align__(16) unsigned char pt_smem_raw[];
  __shared__ __align__(16) uint4 answer_s;
  __shared__ __align__(8) unsigned long long full_s[NS], empty_s[NS], qfull_s[2], qempty_s[2], sfull_s[2], pfull_s[2], odone_s[2], ifull_s[2], iempty_s[2], ask_s, work_s, drain_s;
  __shared__ PtItem item_s[2];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s, beat_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int heads = a.n_kv_heads * a.group, per = by_heads ? heads / 2 : heads;
  const uint32_t smem0 = (smem_u32(pt_smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = smem0, ring = smem0 + 2 * T::kTileBytes;
  volatile int *abort_flag = &abort_s, *beat = &beat_s;

  if (tid == 0) {
#pragma unroll
    for (int i = 0; i < NS; ++i) mbar_init(smem_u32(&full_s[i]), 1), mbar_init(smem_u32(&empty_s[i]), 1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&qfull_s[t]), 1), mbar_init(smem_u32(&qempty_s[t]), 1), mbar_init(smem_u32(&sfull_s[t]), 1), mbar_init(smem_u32(&odone_s[t]), 1);
      mbar_init(smem_u32(&pfull_s[t]), kPtTile);
      mbar_init(smem_u32(&ifull_s[t]), 1), mbar_init(smem_u32(&iempty_s[t]), kPtReaders);
    }
    mbar_init(smem_u32(&ask_s), 1), mbar_init(smem_u32(&work_s), 1), mbar_init(smem_u32(&drain_s), 1);
    abort_s = 0, beat_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // Tensor memory is taken when the kernels before this one are done (none of them then waits for what this one holds), and the ones behind it,
  // which may take theirs before they wait, come after that. (Not needed while no other kernel with tensor memory fits beside this one; 0.2 us a call.)
  griddep_wait();
  if (warp == kPtMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  griddep_launch_dependents();
  auto head_of = [&](const PtItem& w, int t) { return by_heads ? 2 * w.p + t : w.p; };
  auto tok_of = [&](const PtItem& w, int t) { return by_heads ? w.tok0 : w.tok0 + t * kPtTile; };
  // Item k for a reader's warp (false: there is none, or the CTA has given up), and the end of the reading.
  auto take_item = [&](int k) -> bool { return pt_wait(smem_u32(&ifull_s[k & 1]), (k >> 1) & 1, abort_flag, beat) && item_s[k & 1].some != 0; };
  auto give_item = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&iempty_s[k & 1]));
  };
  auto read_item = [&](int k, PtItem& w) -> bool {
    if (!pt_wait_small<D, CAP, BIAS>(smem_u32(&ifull_s[k & 1]), (k >> 1) & 1, abort_flag, beat)) return false;
    w = item_s[k & 1];
    if (w.some == 0) return false;
    give_item(k);
    return true;
  };

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax and output of tile t
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPtSoftRegs));
    const int t = warp >> 2, row = tid & (kPtTile - 1);
    const uint32_t lane_base = tmem + ((uint32_t)(warp & 3) << 21);  // this warp's 32 lanes
    const uint32_t s_t = lane_base + t * kPtTile, o_t = lane_base + 2 * kPtTile + t * D;
    uint32_t blocks = 0, outputs = 0;  // done so far, over all items
    bool ok = true;
    for (int k = 0; ok && take_item(k); ++k) {
      const PtItem& w = item_s[k & 1];  // (read where it is used: registers are short here)
      const int i = tok_of(w, t) + row, head = head_of(w, t), steps = w.je[t] - w.jb[t];
      const int all_from = w.all_from[t], all_to = w.all_to[t];
      int lo, hi, j0 = w.base + w.je[t] * kPtTile;  // the block's first key
      prompt_interval(a, w.s, i, w.n, lo, hi);
      const float slope = BIAS ? a.slopes[head] * kPromptLog2e : 0.f;
      float m = -INFINITY, l = 0.f;
      for (int it = 0; it < steps; ++it, ++blocks) {
        ok = pt_wait(smem_u32(&sfull_s[t]), blocks & 1, abort_flag, beat);
        if (!ok) break;
        tc_fence_after();
        float x[128];
        {
          uint32_t raw[4][32];
#pragma unroll
          for (int c = 0; c < 4; ++c) tc_ld32(s_t + 32 * c, raw[c]);
          tc_wait_ld();
#pragma unroll
          for (int c = 0; c < 128; ++c) x[c] = __uint_as_float(raw[c >> 5][c & 31]);
        }
        const bool edge = it < all_from || it >= all_to;
        j0 -= kPtTile;
        float scale = a.scale_log2;  // from x to log2 units
        if (CAP) {  // x <- tanh(inv x) / inv
          const float inv = a.inv_cap;
          float far[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < 128; c += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) far[e] = pt_max3_abs(far[e], x[c + e], x[c + e + 4]);
          const float most = i < w.n ? pt_max(pt_max(far[0], far[1]), pt_max(far[2], far[3])) * inv : 0.f;  // (rows behind the end hold anything)
          const PtNear near = pt_near(inv);
          if (__builtin_expect(__all_sync(0xFFFFFFFFu, most <= a.near_end), 1)) {
#pragma unroll
            for (int c = 0; c < 128; c += 16) {
              pt2 z[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) z[e] = pt2(x[c + 2 * e], x[c + 2 * e + 1]);
              pt_tanh_near<8>(z, near);
#pragma unroll
              for (int e = 0; e < 8; ++e) z[e].get(x[c + 2 * e], x[c + 2 * e + 1]);
            }
          } else {  // which form an element takes goes by itself: no row depends on its neighbours
            const float back = a.cap_log2 / a.scale_log2;  // 1 / inv
#pragma unroll
            for (int c = 0; c < 128; c += 8) {
              pt2 z[4], y[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) z[e] = pt_mul(pt2(x[c + 2 * e], x[c + 2 * e + 1]), pt2(inv, inv));
              pt_tanh<4>(z);
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] = pt2(x[c + 2 * e], x[c + 2 * e + 1]);
              pt_tanh_near<4>(y, near);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float z0, z1, y0, y1;
                pt_mul(z[e], pt2(back, back)).get(z0, z1), y[e].get(y0, y1);
                const bool n0 = fabsf(x[c + 2 * e] * inv) <= a.near_end, n1 = fabsf(x[c + 2 * e + 1] * inv) <= a.near_end;
                x[c + 2 * e] = n0 ? y0 : z0, x[c + 2 * e + 1] = n1 ? y1 : z1;
              }
            }
          }
        }
        if (BIAS) {
          const float away = (float)(j0 - i);
          const pt2 sc(scale, scale);
          if (a.prefix == nullptr || j0 + kPtTile - 1 <= i - row) {  // no row sees a key behind it
            const pt2 up(8.f * slope, 8.f * slope);
#pragma unroll
            for (int q = 0; q < 128; q += 32) {
              pt2 bias[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) bias[e] = pt2(slope * (away + (float)(q + 2 * e)), slope * (away + (float)(q + 2 * e + 1)));
#pragma unroll
              for (int c = q; c < q + 32; c += 2) {
                const int e = (c >> 1) & 3;
                pt_fma(pt2(x[c], x[c + 1]), sc, bias[e]).get(x[c], x[c + 1]);
                bias[e] = pt_add(bias[e], up);
              }
            }
          } else {
#pragma unroll
            for (int c = 0; c < 128; ++c) x[c] = fmaf(x[c], scale, -slope * fabsf(away + (float)c));
          }
          scale = 1.f;
        }
        if (edge) {
          const uint32_t from = (uint32_t)(lo - j0), span = lo < hi ? (uint32_t)(hi - lo) : 0u;
#pragma unroll
          for (int c = 0; c < 128; ++c) x[c] = (uint32_t)c - from < span ? x[c] : -INFINITY;
        }
        float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 128; c += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e) tops[e] = pt_max3(tops[e], x[c + e], x[c + e + 4]);
        const float top = pt_max(pt_max(tops[0], tops[1]), pt_max(tops[2], tops[3])) * scale;
        const float mx = pt_max(m, top);
        const bool grown = i < w.n && !(mx <= m + kPtSlack);  // (also m = -inf, the first keys that a row sees, and a NaN)
        if (__any_sync(0xFFFFFFFFu, grown)) {
          const float corr = grown ? pt_ex2(m - mx) : 1.f;  // (a row does not depend on its neighbours)
          if (grown) m = mx;
          l *= corr;
          if (it > 0) {  // the product of the block before is done: S of this one was issued behind it
#pragma unroll
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              pt_ld16(o_t + c, o);
              tc_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr);
              pt_st16(o_t + c, o);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.f : m + (m - m);  // (an infinite score: NaN, as inf - inf)
        const pt2 sc(scale, scale), off(-ref, -ref);
        pt2 sum[2] = {pt2(0.f, 0.f), pt2(0.f, 0.f)};
        float p[128] = {};
        uint32_t packed[4][16];
        // Pair e: into the sum, rounded, and every 16 pairs to tensor memory.
        auto finish = [&](int e) {
          sum[e & 1] = pt_add(sum[e & 1], pt2(p[2 * e], p[2 * e + 1]));
          packed[e >> 4][e & 15] = pt_pack(p[2 * e], p[2 * e + 1]);
          if ((e & 15) == 15) pt_st16(s_t + 16 * (e >> 4), packed[e >> 4]);
        };
        // The special-function pipe takes the pairs in a row, sums and rounding follow eight pairs behind; the last EMU pairs go to the FMA pipe.
#pragma unroll
        for (int e = 0; e < 64 - EMU; ++e) {
          pt_fma(pt2(x[2 * e], x[2 * e + 1]), sc, off).get(p[2 * e], p[2 * e + 1]);
          p[2 * e] = pt_ex2(p[2 * e]), p[2 * e + 1] = pt_ex2(p[2 * e + 1]);
          if (e >= 8) finish(e - 8);
        }
        if (EMU > 0) {
          pt2 y[EMU];
#pragma unroll
          for (int e = 0; e < EMU; ++e) y[e] = pt_fma(pt2(x[128 - 2 * EMU + 2 * e], x[128 - 2 * EMU + 2 * e + 1]), sc, off);
          pt_ex2_fma<EMU>(y, p + 128 - 2 * EMU);
          if (edge) {  // (hidden keys weigh exactly nothing)
#pragma unroll
            for (int e = 128 - 2 * EMU; e < 128; ++e) p[e] = x[e] == -INFINITY ? 0.f : p[e];
          }
        }
#pragma unroll
        for (int e = 56 - EMU; e < 64; ++e) finish(e);
        pt_wait_st();
        tc_fence_before();
        mbar_arrive(smem_u32(&pfull_s[t]));
        float s0, s1;
        pt_add(sum[0], sum[1]).get(s0, s1);
        l += s0 + s1;
        if ((it & 63) == 63 && lane == 0) *beat = *beat + 1;
      }
      if (ok && steps > 0) ok = pt_wait(smem_u32(&odone_s[t]), outputs++ & 1, abort_flag, beat);
      if (!ok) break;
      tc_fence_after();
      const float inv = m != -INFINITY ? 1.f / l : 0.f;  // (scores of -inf alone: pt_ex2_fma leaves 2^-125 of their weights)
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + (w.s * a.os[0] + head * a.os[1] + i * a.os[2]);
      const bool none = inv == 0.f;  // (a row that sees nothing: zeros)
      float nan[2] = {0.f, 0.f};     // NaN once an output is
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32] = {};
        if (steps > 0) {
          tc_ld32(o_t + c, o);
          tc_wait_ld();
        }
        uint32_t word[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float f0, f1;
          pt_mul(pt2(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1])), pt2(inv, inv)).get(f0, f1);
          nan[e & 1] = pt_max3(nan[e & 1], f0, f1);
          word[e] = none ? 0u : pt_pack(f0, f1);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i < w.n && c + 8 * e < a.d) *reinterpret_cast<uint4*>(out + c + 8 * e) = make_uint4(word[4 * e], word[4 * e + 1], word[4 * e + 2], word[4 * e + 3]);
      }
      const bool bad = !none && l == l && pt_max(nan[0], nan[1]) != pt_max(nan[0], nan[1]);
      const uint32_t again = __ballot_sync(0xFFFFFFFFu, bad && i < w.n);
      __syncwarp();
      if (again != 0u) prompt_rows_again(a, w.s, head, i - lane, again, w.n, w.base + w.jb[t] * kPtTile, min(w.base + w.je[t] * kPtTile, w.n), beat);
      tc_fence_before();
      give_item(k);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPtOtherRegs));
    if (warp == kPtLoadWarp) {
      // ---------------------------------------------------------------- copies
      uint32_t used = 0, queries[2] = {0, 0};  // K or V tiles and Q tiles asked for so far
      bool ok = true;
      PtItem w;
      for (int k = 0; ok && read_item(k, w); ++k) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (ok && w.je[t] > w.jb[t]) {
            if (queries[t] > 0) ok = pt_wait_small<D, CAP, BIAS>(smem_u32(&qempty_s[t]), (queries[t] - 1) & 1, abort_flag, beat);
            if (!ok) break;
            if (lane == 0) {
              const uint32_t bar = smem_u32(&qfull_s[t]);
              mbar_arrive_expect_tx(bar, T::kTileBytes);
#pragma unroll
              for (int h = 0; h < NH; ++h) tma_load_4d(q_smem + t * T::kTileBytes + h * BOX, &maps.q, 64 * h, tok_of(w, t), head_of(w, t), w.s, bar);
            }
            ++queries[t];
          }
        const int j_begin = w.jb[0] == w.je[0] ? w.jb[1] : w.jb[1] == w.je[1] ? w.jb[0] : min(w.jb[0], w.jb[1]), j_end = max(w.je[0], w.je[1]);
        const int kv = head_of(w, 0) / a.group;
        const int blocks = j_end - j_begin, ask = max(blocks + 1 - kPtAsk, 0);
        int at_key = w.base + j_end * kPtTile;  // of the V block
        if (ok && lane == 0 && blocks == 0) mbar_arrive(smem_u32(&ask_s));
        for (int step = 0; ok && blocks > 0 && step <= blocks; ++step) {
          if (lane == 0 && step == ask) mbar_arrive(smem_u32(&ask_s));
          const uint32_t slot = used % NS;
          if (used >= NS) ok = pt_wait_small<D, CAP, BIAS>(smem_u32(&empty_s[slot]), ((used / NS) - 1) & 1, abort_flag, beat);
          if (!ok) break;
          if (lane == 0) {
            const uint32_t bar = smem_u32(&full_s[slot]), at = ring + slot * 2 * T::kTileBytes;
            mbar_arrive_expect_tx(bar, (step > 0 && step < blocks ? 2u : 1u) * T::kTileBytes);
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              if (step > 0) tma_load_4d(at + T::kTileBytes + h * BOX, &maps.v, 64 * h, at_key, kv, w.s, bar);
              if (step < blocks) tma_load_4d(at + h * BOX, &maps.k, 64 * h, at_key - kPtTile, kv, w.s, bar);
            }
          }
          ++used, at_key -= kPtTile;
        }
      }
      __syncwarp();
      if (__any_sync(0xFFFFFFFFu, *abort_flag != 0)) {  // let what is in flight land before shared memory is given up
        for (int t = 0; t < 2; ++t)
          if (queries[t] > 0) mbar_drain(smem_u32(&qfull_s[t]), (queries[t] - 1) & 1);
        for (uint32_t u = used > (uint32_t)NS ? used - NS : 0; u < used; ++u) mbar_drain(smem_u32(&full_s[u % NS]), (u / NS) & 1);
      }
    } else if (warp == kPtMmaWarp) {
      // ---------------------------------------------------------------- products
      // This warp shares its scheduler's instruction cache with softmax code that is many times larger, and fetches what it runs once a step
      // anew: few instructions count. Hence the elections inside the instructions, the tiles in a loop, one wait and one release a step.
      constexpr uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((kPtTile / 8) << 17) | ((kPtTile / 16) << 24);
      constexpr uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) /* B is MN-major */ | ((D / 8) << 17) | ((kPtTile / 16) << 24);
      const uint64_t qdesc = umma_desc_k128(q_smem), kdesc = umma_desc_k128(ring), vdesc = pt_desc_mn128(ring + T::kTileBytes);
      uint32_t slot = 0, lap = 0, taken = 0, queries = 0;  // ring place of the next step, the parity of its use; parities of the blocks of P and of the Q tiles, a bit a tile
      const uint32_t leader = tc_elect() ? 1u : 0u;
      bool ok = true;
      PtItem w;
      for (int k = 0; ok && read_item(k, w); ++k) {
        const int j_begin = w.jb[0] == w.je[0] ? w.jb[1] : w.jb[1] == w.je[1] ? w.jb[0] : min(w.jb[0], w.jb[1]), j_end = max(w.je[0], w.je[1]);
        if (j_begin == j_end) continue;
#pragma unroll 1
        for (int j = j_end; j >= j_begin; --j) {
          // O += P V of block j, S of block j - 1, tile by tile
          ok = pt_wait_small<D, CAP, BIAS>(smem_u32(&full_s[slot]), lap, abort_flag, beat);
          if (!ok) break;
          const int rows = w.last_rows;  // (of block j_end - 1; all others are full)
          if (__builtin_expect(j + 1 == j_end && rows < kPtTile, 0)) {  // V rows behind the prompt's end hold anything: zeros
            const int chunks = (kPtTile - rows) * 8;
            for (int c = lane; c < chunks * NH; c += 32)
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring + (2 * slot + 1) * T::kTileBytes + (c / chunks) * BOX + rows * 128 + (c % chunks) * 16), "r"(0) : "memory");
            fence_proxy_async();
            __syncwarp();
          }
          const uint64_t at = (uint64_t)(slot * (2 * T::kTileBytes >> 4));
#pragma unroll 1
          for (int t = 0; t < 2; ++t) {
            const int t_begin = t ? w.jb[1] : w.jb[0], t_end = t ? w.je[1] : w.je[0];
            const uint32_t s_at = tmem + t * kPtTile;
            if (j >= t_begin && j < t_end) {
              ok = pt_wait_small<D, CAP, BIAS>(smem_u32(&pfull_s[t]), (taken >> t) & 1, abort_flag, beat);
              if (!ok) break;
              taken ^= 1u << t;
              tc_fence_after();
#pragma unroll
              for (int ks = 0; ks < kPtTile / 16; ++ks)
                pt_mma_ts(leader, tmem + 2 * kPtTile + t * D, s_at + 8 * ks, vdesc + at + (uint64_t)((ks * 16 * 128) >> 4), idesc_pv, ks != 0 || j + 1 != t_end);
              if (j == t_begin) pt_commit(leader, smem_u32(&odone_s[t]));
            }
            if (j > t_begin && j <= t_end) {
              if (j == t_end) {
                ok = pt_wait_small<D, CAP, BIAS>(smem_u32(&qfull_s[t]), (queries >> t) & 1, abort_flag, beat);
                if (!ok) break;
                queries ^= 1u << t;
              }
              const uint64_t ad = qdesc + (uint64_t)(t * (T::kTileBytes >> 4));
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks) {
                const uint64_t of = (uint64_t)(((ks >> 2) * BOX + (ks & 3) * 32) >> 4);
                pt_mma_ss(leader, s_at, ad + of, kdesc + at + of, idesc_qk, ks != 0);
              }
              pt_commit(leader, smem_u32(&sfull_s[t]));
              if (j - 1 == t_begin) pt_commit(leader, smem_u32(&qempty_s[t]));
            }
          }
          if (!ok) break;
          pt_commit(leader, smem_u32(&empty_s[slot]));
          if (++slot == NS) slot = 0, lap ^= 1u;
        }
      }
      if (!ok || __any_sync(0xFFFFFFFFu, *abort_flag != 0)) {  // products in flight end before tensor memory is given up
        pt_commit(leader, smem_u32(&drain_s));
        mbar_drain(smem_u32(&drain_s), 0);
      }
    } else if (warp == kPtWorkWarp) {
      // ---------------------------------------------------------------- work
      const uint32_t answer = smem_u32(&answer_s);
      int cta = blockIdx.x, k = 0;
      uint32_t asked = 0;
      bool ok = true;
      auto hand_over = [&](const PtItem& w) {
        if (k >= 2) ok = ok && pt_wait_small<D, CAP, BIAS>(smem_u32(&iempty_s[k & 1]), ((k >> 1) - 1) & 1, abort_flag, beat);
        if (!ok) return;
        if (lane == 0) {
          item_s[k & 1] = w;
          mbar_arrive(smem_u32(&ifull_s[k & 1]));
        }
        __syncwarp();
        ++k;
      };
      PtItem w;
      while (ok) {
        w.some = 1, w.p = cta % per, w.s = (cta / per) % a.batch;
        const int tile = tiles - 1 - cta / per / a.batch;
        w.tok0 = by_heads ? tile * kPtTile : tile * 2 * kPtTile;
        w.n = min(max(a.lens[w.s], 0), a.tokens);
        if (w.tok0 < w.n) {
          w.base = 0x7FFFFFFF;
          for (int t = 0; t < 2; ++t) {
            int first = 0x7FFFFFFF, end = 0, all_lo = 0, all_hi = 0x7FFFFFFF;  // what its rows see, any and all of them
#pragma unroll 1
            for (int r = 0; r < kPtTile / 32; ++r) {
              const int i = tok_of(w, t) + 32 * r + lane;
              int lo, hi;
              prompt_interval(a, w.s, i, w.n, lo, hi);
              if (lo < hi) first = min(first, lo), end = max(end, hi);
              if (i < w.n) all_lo = max(all_lo, lo < hi ? lo : 0x7FFFFFFF), all_hi = min(all_hi, hi);
            }
            first = __reduce_min_sync(0xFFFFFFFFu, first), end = __reduce_max_sync(0xFFFFFFFFu, end);
            w.all_from[t] = __reduce_min_sync(0xFFFFFFFFu, all_hi), w.all_to[t] = __reduce_max_sync(0xFFFFFFFFu, all_lo);
            w.jb[t] = first, w.je[t] = end, w.base = min(w.base, first);
          }
          w.last_rows = w.n - w.base - (max(w.je[0], w.je[1]) - w.base + kPtTile - 1) / kPtTile * kPtTile + kPtTile;
          for (int t = 0; t < 2; ++t) {
            const bool any = w.je[t] > 0;
            w.jb[t] = any ? (w.jb[t] - w.base) / kPtTile : 0, w.je[t] = any ? (w.je[t] - w.base + kPtTile - 1) / kPtTile : 0;
            w.all_from[t] = w.je[t] - max(w.all_from[t] - w.base, 0) / kPtTile;
            w.all_to[t] = w.je[t] - (int)(((unsigned)(w.all_to[t] - w.base) + kPtTile - 1) / kPtTile);
          }
          hand_over(w);
          // not before this item is nearly done: a CTA that took the next one at once would be bound to it however long this one lasts
          ok = ok && pt_wait_small<D, CAP, BIAS>(smem_u32(&ask_s), (k - 1) & 1, abort_flag, beat);
        }
        if (!ok) break;
        if (lane == 0) pt_ask_work(answer, smem_u32(&work_s));
        ++asked;
        if (!pt_wait_small<D, CAP, BIAS>(smem_u32(&work_s), (asked - 1) & 1, abort_flag, beat)) break;
        const bool more = pt_read_work(answer, cta);
        __syncwarp();  // every lane has read the answer before the next one may be written
        if (!more) {
          w.some = 0;
          hand_over(w);
          break;
        }
      }
      if (asked > 0 && __any_sync(0xFFFFFFFFu, *abort_flag != 0)) mbar_drain(smem_u32(&work_s), (asked - 1) & 1);
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
