// he_attend for any supported dtype and d, and where no tensor map can be encoded: one slot at a time, dot products by warp shuffles;
// and he_attention_loss, which measures what the eviction has dropped.
#pragma once
#include "attend_kernels.cuh"

namespace he {

static __global__ void __launch_bounds__(kAttendThreads) attend_generic_kernel(const AttendArgs a) {
  extern __shared__ __align__(16) float asm_[];  // q as fp32 [G][d], then part_ml [warps][G][2], part_o [warps][G][d]
  const he_config& cfg = a.cfg;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.y * cfg.n_kv_heads + blockIdx.x;
  const int d = cfg.head_dim, G = cfg.group_size, es = esize_of(cfg.dtype);
  const int fill = a.ca.fill[unit];
  float* qs = asm_;
  float* part_ml = qs + G * d;
  float* part_o = part_ml + kAttendWarps * G * 2;
  const int cpr = d * es / 16;
  for (int idx = tid; idx < G * cpr; idx += kAttendThreads)
    stage_chunk(qs + (idx / cpr) * d, static_cast<const char*>(a.q) + ((size_t)unit * G + idx / cpr) * d * es, idx % cpr, cfg.dtype);
  __syncthreads();
  const float scale = rsqrtf((float)d) * kLog2e;
  const char* Kb = static_cast<const char*>(a.ca.k_cache) + (size_t)unit * cfg.max_budget * d * es;
  const char* Vb = static_cast<const char*>(a.ca.v_cache) + (size_t)unit * cfg.max_budget * d * es;
  const int per = d / 32 + (d % 32 ? 1 : 0);  // channels per lane (<= 8): c = lane + 32 * i
  float m[kMaxGroup], l[kMaxGroup], o[kMaxGroup][kMaxDim / 32];
#pragma unroll
  for (int g = 0; g < kMaxGroup; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxDim / 32; ++i) o[g][i] = 0.f;
  }
  auto elem = [&](const char* row, int c) -> float {
    return cfg.dtype == HE_DTYPE_BF16 ? bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(row)[c])
                                      : reinterpret_cast<const float*>(row)[c];
  };
  for (int j = warp; j < fill; j += kAttendWarps) {
    const char* kr = Kb + (size_t)j * d * es;
    const char* vr = Vb + (size_t)j * d * es;
    float kv[kMaxDim / 32], vv[kMaxDim / 32];
#pragma unroll
    for (int i = 0; i < kMaxDim / 32; ++i) {
      const int c = lane + 32 * i;
      kv[i] = (i < per && c < d) ? elem(kr, c) : 0.f;
      vv[i] = (i < per && c < d) ? elem(vr, c) : 0.f;
    }
#pragma unroll
    for (int g = 0; g < kMaxGroup; ++g) {
      if (g < G) {
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < kMaxDim / 32; ++i) {
          const int c = lane + 32 * i;
          if (i < per && c < d) dot = fmaf(qs[g * d + c], kv[i], dot);
        }
        for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, off);
        const float sc = dot * scale;
        const float mn = fmaxf(m[g], sc), ref = mn == -INFINITY ? 0.f : mn;    // (scores of -inf alone so far: no weight)
        const float corr = exp2f(m[g] - ref), p = exp2f(sc - ref);  // exp2f(-inf) = 0 on the first slot
        l[g] = l[g] * corr + p;
#pragma unroll
        for (int i = 0; i < kMaxDim / 32; ++i) o[g][i] = o[g][i] * corr + p * vv[i];
        m[g] = mn;
      }
    }
  }
#pragma unroll
  for (int g = 0; g < kMaxGroup; ++g) {
    if (g < G) {
      if (lane == 0) {
        part_ml[(warp * G + g) * 2] = m[g];
        part_ml[(warp * G + g) * 2 + 1] = l[g];
      }
#pragma unroll
      for (int i = 0; i < kMaxDim / 32; ++i) {
        const int c = lane + 32 * i;
        if (i < per && c < d) part_o[(warp * G + g) * d + c] = o[g][i];
      }
    }
  }
  __syncthreads();
  attend_merge<kAttendWarps>(part_ml, part_o, G, d, a.out + (size_t)unit * G * d);
}

// ------------------------------------------------------------------------------------------------ attention loss
//
// he_attention_loss (Section 4.6 / Appendix B): 1 - the attention mass of the cached tokens, for each query head, under
// softmax(q . k_p / sqrt(d)) over ALL n = next_pos tokens seen so far. The dropped mass is summed directly (a token
// is dropped when no valid slot holds its position: a bitmap in shared memory), so a small loss is not the
// difference of two numbers close to one. One CTA per unit, a warp per token, online maximum as in he_attend.
struct LossArgs {
  he_config cfg;
  he_cache ca;
  const void* q;       // [B, Hkv*G, d]
  const void* k_full;  // strided [B, Hkv, n, d]
  long long s0, s1, s2;
  float* out;          // [B, Hkv*G]
};

static __global__ void __launch_bounds__(kAttendThreads) attention_loss_kernel(const LossArgs a) {
  extern __shared__ __align__(16) float lsm_[];  // q as fp32 [G][d], partials [warps][G][3], bitmap of cached positions
  const he_config& cfg = a.cfg;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long unit = (long long)blockIdx.y * cfg.n_kv_heads + blockIdx.x;
  const int d = cfg.head_dim, G = cfg.group_size, es = esize_of(cfg.dtype);
  const int n = a.ca.next_pos[unit], fill = a.ca.fill[unit];
  float* qs = lsm_;
  float* part = qs + G * d;
  uint32_t* kept = reinterpret_cast<uint32_t*>(part + kAttendWarps * G * 3);
  const int cpr = d * es / 16;
  for (int idx = tid; idx < G * cpr; idx += kAttendThreads)
    stage_chunk(qs + (idx / cpr) * d, static_cast<const char*>(a.q) + (unit * G + idx / cpr) * d * es, idx % cpr, cfg.dtype);
  for (int i = tid; i < (n + 31) / 32; i += kAttendThreads) kept[i] = 0u;
  __syncthreads();
  for (int j = tid; j < fill; j += kAttendThreads) {
    const int p = a.ca.pos[unit * cfg.max_budget + j];
    if (p >= 0 && p < n) atomicOr(&kept[p >> 5], 1u << (p & 31));
  }
  __syncthreads();
  const float scale = rsqrtf((float)d) * kLog2e;
  const char* Kb = static_cast<const char*>(a.k_full) + ((long long)blockIdx.y * a.s0 + (long long)blockIdx.x * a.s1) * es;
  float m[kMaxGroup], lall[kMaxGroup], ldrop[kMaxGroup];
#pragma unroll
  for (int g = 0; g < kMaxGroup; ++g) m[g] = -INFINITY, lall[g] = 0.f, ldrop[g] = 0.f;
  const int per = (d + 31) / 32;
  for (int p = warp; p < n; p += kAttendWarps) {
    const char* kr = Kb + (long long)p * a.s2 * es;
    float kv[kMaxDim / 32];
#pragma unroll
    for (int i = 0; i < kMaxDim / 32; ++i) {
      const int c = lane + 32 * i;
      kv[i] = (i < per && c < d) ? (cfg.dtype == HE_DTYPE_BF16 ? bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(kr)[c])
                                                                : reinterpret_cast<const float*>(kr)[c])
                                 : 0.f;
    }
    const bool dropped = ((kept[p >> 5] >> (p & 31)) & 1u) == 0u;
#pragma unroll
    for (int g = 0; g < kMaxGroup; ++g) {
      if (g < G) {
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < kMaxDim / 32; ++i) {
          const int c = lane + 32 * i;
          if (i < per && c < d) dot = fmaf(qs[g * d + c], kv[i], dot);
        }
        for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, off);
        const float sc = dot * scale;
        const float mn = fmaxf(m[g], sc);
        const float corr = exp2f(m[g] - mn), w = exp2f(sc - mn);
        lall[g] = lall[g] * corr + w;
        ldrop[g] = ldrop[g] * corr + (dropped ? w : 0.f);
        m[g] = mn;
      }
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int g = 0; g < kMaxGroup; ++g)
      if (g < G) {
        part[(warp * G + g) * 3] = m[g];
        part[(warp * G + g) * 3 + 1] = lall[g];
        part[(warp * G + g) * 3 + 2] = ldrop[g];
      }
  }
  __syncthreads();
  if (tid < G) {
    float M = -INFINITY;
    for (int w = 0; w < kAttendWarps; ++w) M = fmaxf(M, part[(w * G + tid) * 3]);
    float A = 0.f, D = 0.f;
    for (int w = 0; w < kAttendWarps; ++w) {
      const float mw = part[(w * G + tid) * 3];
      const float f = mw == -INFINITY ? 0.f : exp2f(mw - M);
      A += part[(w * G + tid) * 3 + 1] * f;
      D += part[(w * G + tid) * 3 + 2] * f;
    }
    a.out[unit * G + tid] = A > 0.f ? D / A : 0.f;
  }
}

// The same for bf16 keys with d = 128 and G <= 8: scores of 16 tokens at a time as warp-level MMAs fed straight from
// 16-byte global loads (the fragment scheme of attend_bf16_kernel), next group's rows requested before the current
// group's arithmetic. Dynamic shared memory: partials [warps][G][3] floats, then the bitmap of cached positions.
static __global__ void __launch_bounds__(kAttendThreads) attention_loss_bf16_kernel(const LossArgs a) {
  extern __shared__ __align__(16) float lsm_[];
  constexpr int d = 128;
  const he_config& cfg = a.cfg;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const long long unit = (long long)blockIdx.y * cfg.n_kv_heads + blockIdx.x;
  const int G = cfg.group_size;
  const int n = a.ca.next_pos[unit], fill = a.ca.fill[unit];
  float* part = lsm_;
  uint32_t* kept = reinterpret_cast<uint32_t*>(part + kAttendWarps * G * 3);
  for (int i = tid; i < (n + 31) / 32; i += kAttendThreads) kept[i] = 0u;
  __syncthreads();
  for (int j = tid; j < fill; j += kAttendThreads) {
    const int p = a.ca.pos[unit * cfg.max_budget + j];
    if (p >= 0 && p < n) atomicOr(&kept[p >> 5], 1u << (p & 31));
  }
  __syncthreads();
  uint32_t qf[8][2];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint4 t = make_uint4(0u, 0u, 0u, 0u);
    if (gid < G) t = static_cast<const uint4*>(a.q)[(unit * G + gid) * (d / 8) + tig + 4 * c];
    qf[2 * c][0] = t.x, qf[2 * c][1] = t.y, qf[2 * c + 1][0] = t.z, qf[2 * c + 1][1] = t.w;
  }
  const float scale = rsqrtf((float)d) * kLog2e;
  const char* Kb = static_cast<const char*>(a.k_full) + ((long long)blockIdx.y * a.s0 + (long long)blockIdx.x * a.s1) * 2;
  const int last = n - 1;
  auto load_k = [&](int g0, uint4 (&kb)[2][4]) {  // rows past the end repeat the last row and are weighted by zero
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint4* row = reinterpret_cast<const uint4*>(Kb + (long long)min(g0 + gid + 8 * r, last) * a.s2 * 2);
#pragma unroll
      for (int c = 0; c < 4; ++c) kb[r][c] = ldg_stream16(row + tig + 4 * c);
    }
  };
  float m = -INFINITY, lall = 0.f, ldrop = 0.f;
  uint4 kc[2][4], kn[2][4];
  const int stride = 16 * kAttendWarps;
  int g0 = 16 * warp;
  if (g0 < n) load_k(g0, kc);
  for (; g0 < n; g0 += stride) {
    const bool more = g0 + stride < n;
    if (more) load_k(g0 + stride, kn);
    float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      mma_bf16_m16n8k16(s0, qf[2 * c][0], 0u, qf[2 * c][1], 0u, kc[0][c].x, kc[0][c].y);
      mma_bf16_m16n8k16(s1, qf[2 * c][0], 0u, qf[2 * c][1], 0u, kc[1][c].x, kc[1][c].y);
      mma_bf16_m16n8k16(s0, qf[2 * c + 1][0], 0u, qf[2 * c + 1][1], 0u, kc[0][c].z, kc[0][c].w);
      mma_bf16_m16n8k16(s1, qf[2 * c + 1][0], 0u, qf[2 * c + 1][1], 0u, kc[1][c].z, kc[1][c].w);
    }
    // this lane: head gid, tokens g0 + 2tig, + 1, + 8, + 9
    const int j = g0 + 2 * tig;
    const int tok[4] = {j, j + 1, j + 8, j + 9};
    const float sc[4] = {s0[0], s0[1], s1[0], s1[1]};
    float x[4];
    bool dropped[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = tok[e] < n ? sc[e] * scale : -INFINITY;
      dropped[e] = tok[e] < n && ((kept[tok[e] >> 5] >> (tok[e] & 31)) & 1u) == 0u;
    }
    float gm = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 1));
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 2));  // finite: token g0 exists
    const float mn = fmaxf(m, gm);
    const float corr = exp2f(m - mn);
    float wa = 0.f, wd = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float w = exp2f(x[e] - mn);
      wa += w;
      wd += dropped[e] ? w : 0.f;
    }
    lall = lall * corr + wa;
    ldrop = ldrop * corr + wd;
    m = mn;
    if (more) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) kc[r][c] = kn[r][c];
    }
  }
  lall += __shfl_xor_sync(0xFFFFFFFFu, lall, 1);
  lall += __shfl_xor_sync(0xFFFFFFFFu, lall, 2);
  ldrop += __shfl_xor_sync(0xFFFFFFFFu, ldrop, 1);
  ldrop += __shfl_xor_sync(0xFFFFFFFFu, ldrop, 2);
  if (gid < G && tig == 0) {
    part[(warp * G + gid) * 3] = m;
    part[(warp * G + gid) * 3 + 1] = lall;
    part[(warp * G + gid) * 3 + 2] = ldrop;
  }
  __syncthreads();
  if (tid < G) {
    float M = -INFINITY;
    for (int w = 0; w < kAttendWarps; ++w) M = fmaxf(M, part[(w * G + tid) * 3]);
    float A = 0.f, D = 0.f;
    for (int w = 0; w < kAttendWarps; ++w) {
      const float mw = part[(w * G + tid) * 3];
      const float f = mw == -INFINITY ? 0.f : exp2f(mw - M);
      A += part[(w * G + tid) * 3 + 1] * f;
      D += part[(w * G + tid) * 3 + 2] * f;
    }
    a.out[unit * G + tid] = A > 0.f ? D / A : 0.f;
  }
}

}  // namespace he
