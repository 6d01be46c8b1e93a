// he_attend: Eq. 1 over the compressed cache (Algorithm 1 line 6), the step that follows the eviction:
//   out[g] = sum_j softmax_j(q_g . K_j / sqrt(d)) V_j   over the valid slots of the query head's KV unit.
// All G query heads of a group are served together, so K and V are read once for the group. Each warp walks its
// own slots with an online softmax (running maximum, running sum, unnormalised output) and the partial results are
// merged through shared memory at the end. HBM-bound by design: 2 * C * d * e bytes per unit.
//
//   attend_bf16_kernel<D, NW>  bf16, d = 64 or 128, G <= 8: 32 slots at a time from rings of TMA tiles, Q K^T and P V as warp-level
//                          m16n8k16 MMAs (bf16 products are exact, fp32 accumulation, P as hi + lo bf16); a cluster of up
//                          to 16 CTAs shares a unit when there are few units.
//   attend_generic_kernel  any supported dtype / d, and where no tensor map can be encoded (attend_generic_kernels.cuh).
//   attend_scored_kernel   the same for he_attend_scored.
#pragma once
#include <cuda.h>  // CUtensorMap (types only; the encoder is fetched through the runtime)

#include <type_traits>

#include "common.cuh"

namespace he {

// he_score_mod on the device (he_attend_scored): scores in log2 units, cap = 0 and window = 0 for none.
struct AttendMod {
  float scale_log2, cap_log2, inv_cap;  // x = scale_log2 * q.k, or cap_log2 * tanh(inv_cap * q.k)
  int window;
  const float* slopes;       // [Hkv*G] or null
  const int32_t* first_pos;  // [B] or null
};

struct AttendArgs {
  he_config cfg;
  he_cache ca;
  const void* q;  // [B, Hkv*G, d]
  float* out;     // [B, Hkv*G, d] fp32
  AttendMod mod;  // read by the kernels with MOD only
};
struct ScoredArgs : AttendArgs {
  int n_order;  // > 0: the sequences in the order in which their CTAs start, largest budgets first
  uint8_t order[256];
};
template <bool MOD>
using AttendArgsOf = std::conditional_t<MOD, ScoredArgs, AttendArgs>;

constexpr int kAttendThreads = 256;
constexpr int kAttendWarps = kAttendThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

// Merge of the per-warp partial results (m = running max in log2 units, l = running sum, o = unnormalised output).
// part_ml: [warps][G][2], part_o: [warps][G][d]. Every thread writes some of the G * d outputs.
// A sum of zero means that nothing was seen. A score that is a NaN or +inf leaves the sum a NaN (the maxima let a NaN pass by), and the output too.
template <int NW>
__device__ __forceinline__ void attend_merge(const float* part_ml, const float* part_o, int G, int d, float* out_unit) {
  for (int idx = threadIdx.x; idx < G * d; idx += 32 * NW) {
    const int g = idx / d, c = idx % d;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, part_ml[(w * G + g) * 2]);
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float m = part_ml[(w * G + g) * 2];
      const float f = m == -INFINITY ? 0.f : exp2f(m - M);
      L += part_ml[(w * G + g) * 2 + 1] * f;
      O += part_o[(w * G + g) * d + c] * f;
    }
    out_unit[idx] = L != 0.f ? O / L : 0.f;
  }
}

// A cluster of S CTAs on one unit: CTA r > 0 folds its warps and sends the result (G maxima, G sums, G * d outputs) to CTA 0 as
// asynchronous remote stores that count on CTA 0's mbarrier; CTA 0 folds its own into place 0 of `gather`, waits and
// combines. One way across the cluster, no barrier at the end. (Two cluster barriers around remote reads cost 4 us a call
// with 8 CTAs, as much as the streaming of 5 MB per cluster.) The wait is bounded; on a time-out the unit's output is
// undefined and the device error counter is raised.
__device__ __forceinline__ uint32_t attend_mapa(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
constexpr uint32_t kAttendSpinLimit = 1u << 22;
template <int NW>
__device__ __forceinline__ void attend_merge_cluster(const float* part_ml, const float* part_o, float* gather, uint32_t bar, int G,
                                                     int d, int S, int rank, float* out_unit) {
  const int per = G * (d + 2);  // floats of one CTA's result: [G] maxima, [G] sums, [G][d] outputs
  for (int idx = threadIdx.x; idx < G * d; idx += 32 * NW) {
    const int g = idx / d, c = idx % d;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, part_ml[(w * G + g) * 2]);
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float m = part_ml[(w * G + g) * 2];
      const float f = m == -INFINITY ? 0.f : exp2f(m - M);
      L += part_ml[(w * G + g) * 2 + 1] * f;
      O += part_o[(w * G + g) * d + c] * f;
    }
    if (rank == 0) {
      if (c == 0) gather[g] = M, gather[G + g] = L;
      gather[2 * G + idx] = O;
    } else {
      const uint32_t dst = attend_mapa((uint32_t)__cvta_generic_to_shared(gather + rank * per), 0u), rb = attend_mapa(bar, 0u);
      auto send = [&](int at, float v) {
        asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(dst + 4u * at), "r"(__float_as_uint(v)), "r"(rb)
                     : "memory");
      };
      if (c == 0) send(g, M), send(G + g, L);
      send(2 * G + idx, O);
    }
  }
  if (rank != 0) return;
  bool ok = false;
  for (uint32_t i = 0; i < kAttendSpinLimit && !ok; ++i) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], 0;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar)
        : "memory");
    ok = done != 0;
  }
  if (!ok && threadIdx.x == 0) atomicAdd(&g_tc_error, 1);
  __syncthreads();
  for (int idx = threadIdx.x; idx < G * d; idx += 32 * NW) {
    const int g = idx / d;
    float M = -INFINITY;
#pragma unroll 4
    for (int r = 0; r < S; ++r) M = fmaxf(M, gather[r * per + g]);
    float L = 0.f, O = 0.f;
#pragma unroll 4
    for (int r = 0; r < S; ++r) {
      const float m = gather[r * per + g];
      const float f = m == -INFINITY ? 0.f : exp2f(m - M);
      L += gather[r * per + G + g] * f;
      O += gather[r * per + 2 * G + idx] * f;
    }
    out_unit[idx] = L != 0.f ? O / L : 0.f;
  }
}

// ------------------------------------------------------------------------------------------------ bf16, d = 64 or 128
//
// A warp takes 32 slots at a time. Scores: S[head][slot] = Q K^T as m16n8k16 MMAs with M = query heads (rows 0..7
// used), N = 8 slots, K = 16 channels. A dot product does not depend on the order of its terms, so the 16 "logical"
// channels of MMA step s are chosen to suit 16-byte reads: lane (gid, tig) reads chunks 2 tig and 2 tig + 1 (8 channels each) of
// every 64 channels of row gid; the c-th of them feeds steps 2c (first two registers) and 2c+1 (last two); the
// query fragment is loaded the same way, so both operands agree on the permutation.
// Output: O[head][channel] += P V with M = heads, K = 16 slots, N = 8 channels. The score tile's accumulator layout
// is already the A-fragment layout of P (head gid, slots 2tig, 2tig+1 [+8]). P is split into two bf16 terms
// (p = hi + lo + O(2^-18 p)): hi in rows 0..7, lo in rows 8..15 of the same MMA, summed at the end, so that the
// rows a group of <= 8 heads leaves empty carry the low-order term. The B fragment wants pairs of slots per
// channel: lane (gid, tig) holds slots 2tig, 2tig+1, 2tig+8, 2tig+9 and chunks gid, gid+8 of each, and a byte
// permute pairs the two slots' values of one channel. Output tile t = 8h + e of lane column n is channel
// (n + 8h) * 8 + e.

__device__ __forceinline__ void mma_bf16_m16n8k16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                  uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// (hi, lo) bf16 pairs of two fp32 values: hi = round-to-nearest bf16, lo = bf16 of the exact remainder.
// The first value goes to the low half (the lower k index of the fragment).
__device__ __forceinline__ void split_pair(float x, float y, uint32_t& hi, uint32_t& lo) {
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(hi) : "f"(y), "f"(x));
  const float xr = x - __uint_as_float(hi << 16), yr = y - __uint_as_float(hi & 0xFFFF0000u);
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(lo) : "f"(yr), "f"(xr));
}

__device__ __forceinline__ uint4 ldg_stream16(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// K and V rows travel through shared memory as TMA tile copies, a warp's 32-slot groups as a ring of items K0, V0, K1, V1, ...
// that only this warp asks for and reads (an mbarrier per ring buffer, no block barrier). What bounds the call is bytes in
// flight: HBM's latency under load times its bandwidth is about 8 MB, 55 KB per SM, and registers alone hold half of it
// next to the accumulators; the rings keep 128 KB in flight. Calls with few units are bound by what one SM pulls: 16-byte
// cp.async copies into the same rings reached 28 bytes a cycle. The 128-byte swizzle puts chunk c of row r at c ^ (r & 7), and
// the fragment reads below are chosen to meet every bank once: a K read takes the even or the odd chunks of two
// neighbouring rows, a V read two neighbouring chunks of rows r, r + 2, r + 4, r + 6.
//
// Eight warps per SM: NW = 8 is one CTA per SM, for grids that do not fill the SMs twice; NW = 4 two, so that one streams while
// the other starts or merges.
//
// Grid (Hkv * S, B) in clusters of S CTAs along x: the S CTAs of a cluster share one unit's slots (32-slot groups
// dealt round-robin over the S * NW warps), each merges its own warps, and the cluster merges the S partial results
// through distributed shared memory, so a call with few units still fills the GPU without any scratch in HBM.
// Launched with the programmatic-serialization attribute: set-up overlaps the tail of the stream's previous kernel (usually
// the decode step), everything the caller or that kernel wrote is read after the wait.
// Dynamic shared memory: the warps' rings, reused by part_ml [warps][G][2], part_o [warps][G][d]; then, with S > 1, the S CTAs'
// partial results (CTA 0's are used), which may arrive while the rings are still in use.
constexpr int kAttendGroup = 32;  // slots per item
template <int D, int NW>
struct AttendRing {
  static constexpr int kBufs = 3 * (128 / D);  // items in a warp's ring: one being read, the others in flight
  static constexpr int kItemBytes = kAttendGroup * D * 2;
  static constexpr int kBytes = NW * kBufs * kItemBytes;  // 24 KB per warp
};

// With MOD the scores go through he_score_mod: four more bytes a slot (its position, fetched a group ahead into registers) beside 4 D
// of K and V, and masked slots' V rows are cleared in registers, as they may hold anything. With BELOW d is below D: the tensor maps fill the channels
// from d on with zeros.
// Exactness: weights of few slots show the 2^-18 that two bf16 terms leave of each (1.3e-6 of the output at 20 slots), sums over many slots the truncation
// of the MMA's accumulator (1.7e-6 at 8000). With MOD a weight has a third term and each group's products start from zero and are added with rounding: 2e-7 and
// 6e-7. Groups of up to 4 heads (FOLD) hold the third terms in the rows that they leave empty (rows 4..7 repeat the heads of rows 0..3), larger
// ones take products of their own.
// Measured, d = 128 and G = 4: 512 units of 512 to 4096 slots 85.6 us without modification (6.6 TB/s), 86.2 with a cap, a window or slopes: bound by
// HBM (94.5 and 97 with the units in their own order; he_attend 91). 8 units of 9830 slots 11.0 us (he_attend 10.1), 11.9 with a cap: HBM needs 6.3, and a call with clusters pays 4 us
// whatever it reads. Rows that a mask hides are copied like the others (with a window of 1024 over 9830 slots a call from Python takes 12.7 us, without 12.0). Groups of 8 without room
// for the third terms: 128 units of 2048 slots at d = 64 13.6 us (he_attend 10.8), bound by the issue of MMAs and their operands.
template <int D, int NW, bool MOD, bool CAP = false, bool FOLD = false, bool BELOW = false>
__global__ void __launch_bounds__(32 * NW, 8 / NW) attend_bf16_kernel(const AttendArgsOf<MOD> a, const int S, const __grid_constant__ CUtensorMap kmap,
                                                                     const __grid_constant__ CUtensorMap vmap) {
  using Ring = AttendRing<D, NW>;
  extern __shared__ __align__(16) unsigned char attend_smem_raw[];
  __shared__ __align__(8) unsigned long long merge_bar, ring_bar[NW][Ring::kBufs];
  constexpr int CPR = D / 8;               // 16-byte chunks per row in a ring buffer
  constexpr int NC = D / 32, NH = D / 64;  // chunks of a K row per lane, of a V row per lane
  constexpr int NBUF = Ring::kBufs, GRP = kAttendGroup;
  const he_config& cfg = a.cfg;
  const int d = BELOW ? cfg.head_dim : D;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const int rank = blockIdx.x % S;
  int seq = blockIdx.y;
  if constexpr (MOD && NW == 4) seq = a.n_order > 0 ? a.order[blockIdx.y] : seq;
  const int unit = seq * cfg.n_kv_heads + blockIdx.x / S;
  const int G = cfg.group_size;
  // rounded up to 1024 bytes (the swizzle's period) by an offset from the array itself
  float* asm_ = reinterpret_cast<float*>(attend_smem_raw + ((1024u - ((uint32_t)__cvta_generic_to_shared(attend_smem_raw) & 1023u)) & 1023u));
  float* part_ml = asm_;
  float* part_o = part_ml + NW * G * 2;
  float* gather = asm_ + Ring::kBytes / 4;
  const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&merge_bar);
  unsigned char* ring = reinterpret_cast<unsigned char*>(asm_) + warp * NBUF * Ring::kItemBytes;
  auto full = [&](int b) { return (uint32_t)__cvta_generic_to_shared(&ring_bar[warp][b]); };

  griddep_launch_dependents();
  if (lane == 0) {
#pragma unroll
    for (int b = 0; b < NBUF; ++b) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(full(b)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (S > 1) {
    if (rank == 0 && tid == 0) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)((S - 1) * G * (d + 2) * 4)) : "memory");
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // waited for before the first remote store
  }
  const int stride = GRP * NW * S, first = GRP * (warp * S + rank);
  // Where the grid is one wave, each warp's first rows are asked into L2 while the stream's previous kernel (usually the decode step,
  // which moves little) runs: a prefetch returns no data, so it cannot see a stale row. (fill is a hint here: read again below, past
  // L1.) 8 units of 9830 slots behind a decode step: 14.9 us for both without, 14.1 with one group per warp, 14.2 with two, 15.0
  // with three, which the copy engine has not worked off when the wait returns.
  if (NW == 8 && lane == 0) {
    const int rows = min(min(__ldcg(a.ca.fill + unit), cfg.max_budget) - first, GRP);
    const size_t at = ((size_t)unit * cfg.max_budget + first) * d * 2;
    if (rows > 0) {
      l2_prefetch_bulk(static_cast<const char*>(a.ca.k_cache) + at, (uint32_t)rows * d * 2);
      l2_prefetch_bulk(static_cast<const char*>(a.ca.v_cache) + at, (uint32_t)rows * d * 2);
    }
  }
  griddep_wait();
  const int fill = __ldcg(a.ca.fill + unit);
  const int my_head = FOLD ? gid & 3 : gid;
  float slope = 0.f;              // MOD: log2 units per position
  int now = 0, low = 0;           // MOD: the query's position, the first one it sees
  if (MOD) {                      // (asked for together with `fill`, looked at behind the first copies)
    now = __ldcg(a.ca.next_pos + unit) - 1;
    if (a.mod.first_pos != nullptr) low = a.mod.first_pos[seq];
    if (a.mod.slopes != nullptr && my_head < G) slope = a.mod.slopes[(unit % cfg.n_kv_heads) * G + my_head] * kLog2e;
  }
  const int items = first < fill ? 2 * ((fill - first + stride - 1) / stride) : 0;
  const int row_base = unit * cfg.max_budget;
  // Item t (K rows of group t / 2, or its V rows) into buffer b.
  auto issue = [&](int t, int b) {
    if (t < items && lane == 0) {
      const int row = row_base + first + (t >> 1) * stride;
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(ring + b * Ring::kItemBytes);
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full(b)), "r"((uint32_t)Ring::kItemBytes) : "memory");
#pragma unroll
      for (int h = 0; h < NH; ++h)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst + h * GRP * 128),
            "l"(reinterpret_cast<uint64_t>((t & 1) ? &vmap : &kmap)), "r"(h * 64), "r"(row), "r"(full(b))
            : "memory");
    }
  };
#pragma unroll
  for (int t = 0; t < NBUF - 1; ++t) issue(t, t);

  uint32_t qf[2 * NC][2];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    uint4 t = make_uint4(0u, 0u, 0u, 0u);
    const int chunk = 2 * tig + (c & 1) + 8 * (c >> 1);
    if (my_head < G && (!BELOW || chunk < d / 8)) t = static_cast<const uint4*>(a.q)[((size_t)unit * G + my_head) * (d / 8) + chunk];
    qf[2 * c][0] = t.x, qf[2 * c][1] = t.y, qf[2 * c + 1][0] = t.z, qf[2 * c + 1][1] = t.w;
  }
  const float scale = MOD ? a.mod.scale_log2 : rsqrtf((float)d) * kLog2e;
  const int32_t* slot_pos = a.ca.pos + (size_t)unit * cfg.max_budget + 2 * tig;
  int2 ahead[4];  // positions of this lane's slots 8 i + 2 tig, + 1 of the next group
  auto fetch_pos = [&](int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) ahead[i] = g + 8 * i + 2 * tig < fill ? __ldcg(reinterpret_cast<const int2*>(slot_pos + g + 8 * i)) : make_int2(-1, -1);
  };
  if (MOD) {
    fetch_pos(first);
    low = max(low, a.mod.window > 0 ? max(0, now - a.mod.window + 1) : 0);
  }
  float m = -INFINITY, l = 0.f;
  float o[8 * NH][4];
#pragma unroll
  for (int t = 0; t < 8 * NH; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
  int buf = 0;
  uint32_t phase = 0;
  bool ok = true;
  // the next item has landed; its predecessor's buffer, read by the whole warp, takes the item NBUF - 1 ahead
  auto step = [&](int t) -> const uint4* {
    bool got = false;
    for (uint32_t i = 0; ok && i < kAttendSpinLimit && !got; ++i) {
      uint32_t done;
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(done)
          : "r"(full(buf)), "r"(phase)
          : "memory");
      got = done != 0;
    }
    ok = __all_sync(0xFFFFFFFFu, got);
    if (ok) issue(t + NBUF - 1, buf == 0 ? NBUF - 1 : buf - 1);
    const uint4* p = reinterpret_cast<const uint4*>(ring + buf * Ring::kItemBytes);
    if (++buf == NBUF) buf = 0, phase ^= 1u;
    return p;
  };
  for (int t = 0; t < items && ok; t += 2) {
    const int g0 = first + (t >> 1) * stride;
    // scores of slots g0 + 8 i + (0..7): two accumulators each (the chunks' two halves), so no chain is longer than NC
    float sa[4][4], sb[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sa[i][e] = sb[i][e] = 0.f;
    {
      const uint4* kr = step(t) + gid * 8;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // (row 8 i + gid of the half of the channels that holds chunk c)
          const uint4 kv = kr[(c >> 1) * GRP * 8 + i * 64 + ((2 * tig + (c & 1)) ^ gid)];
          mma_bf16_m16n8k16(sa[i], qf[2 * c][0], 0u, qf[2 * c][1], 0u, kv.x, kv.y);
          mma_bf16_m16n8k16(sb[i], qf[2 * c + 1][0], 0u, qf[2 * c + 1][1], 0u, kv.z, kv.w);
        }
    }
    // This lane: head gid, slots g0 + 8 i + 2 tig, + 1.
    float x[8];
    float gm = -INFINITY;
    uint32_t seen = 0u;  // MOD: the group's visible slots
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = 8 * i + 2 * tig + e;
        bool ok_j = g0 + j < fill;
        float s = (sa[i][e] + sb[i][e]) * scale;
        if (MOD) {
          const int p = e ? ahead[i].y : ahead[i].x;
          if (CAP) s = a.mod.cap_log2 * tanhf((sa[i][e] + sb[i][e]) * a.mod.inv_cap);
          s -= slope * (float)abs(now - p);
          ok_j = ok_j && p >= low;
          seen |= (uint32_t)ok_j << j;
        }
        x[2 * i + e] = ok_j ? s : -INFINITY;
        gm = fmaxf(gm, x[2 * i + e]);
      }
    if (MOD) {
      seen = __reduce_or_sync(0xFFFFFFFFu, seen);
      if (t + 2 < items) fetch_pos(g0 + stride);
    }
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 1));
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 2));
    const float mx = fmaxf(m, gm);
    const float mn = mx == -INFINITY ? 0.f : mx;  // (nothing seen so far, or scores of -inf alone: all weights are exp2(-inf))
    const float corr = exp2f(m - mn);
    float p[8], ps = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = exp2f(x[k] - mn);
#pragma unroll
    for (int k = 0; k < 8; k += 2) ps += p[k] + p[k + 1];
    l = l * corr + ps;
    m = mx;
    uint32_t w[4][2];  // hi and lo halves of the weights of slots 8 i + 2 tig, + 1
#pragma unroll
    for (int i = 0; i < 4; ++i) split_pair(p[2 * i], p[2 * i + 1], w[i][0], w[i][1]);
    uint32_t third[4];  // MOD: what two terms leave of a weight
#pragma unroll
    for (int i = 0; MOD && i < 4; ++i) {
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n"
          : "=r"(third[i])
          : "f"(p[2 * i + 1] - __uint_as_float(w[i][0] & 0xFFFF0000u) - __uint_as_float(w[i][1] & 0xFFFF0000u)),
            "f"(p[2 * i] - __uint_as_float(w[i][0] << 16) - __uint_as_float(w[i][1] << 16)));
      if (FOLD && gid >= 4) w[i][0] = third[i], w[i][1] = 0u;
    }
    if (__any_sync(0xFFFFFFFFu, corr != 1.f)) {
#pragma unroll
      for (int t2 = 0; t2 < 8 * NH; ++t2) o[t2][0] *= corr, o[t2][1] *= corr, o[t2][2] *= corr, o[t2][3] *= corr;
    }
    const uint4* vr = step(t + 1);
    if (!MOD && g0 + GRP > fill) {  // rows past the fill level (weighted by zero) hold anything: make them finite
      for (int i = lane; i < GRP * CPR; i += 32)
        if (g0 + ((i >> 3) & (GRP - 1)) >= fill) const_cast<uint4*>(vr)[i] = make_uint4(0u, 0u, 0u, 0u);
      __syncwarp();
    }
    if constexpr (MOD) {
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        uint4 vb[2][4];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int row = 16 * hf + 2 * tig + (s & 1) + 8 * (s >> 1);
            vb[hf][s] = vr[h * GRP * 8 + row * 8 + (gid ^ (row & 7))];
          }
        if (seen != 0xFFFFFFFFu) {  // hidden rows (weighted by zero) hold anything: zeros
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
              const uint32_t keep = 0u - ((seen >> (16 * hf + 2 * tig + (s & 1) + 8 * (s >> 1))) & 1u);
              vb[hf][s].x &= keep, vb[hf][s].y &= keep, vb[hf][s].z &= keep, vb[hf][s].w &= keep;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const uint32_t sel = (e & 1) ? 0x7632u : 0x5410u;
            auto word = [&](const uint4& v) { return (e >> 1) == 0 ? v.x : (e >> 1) == 1 ? v.y : (e >> 1) == 2 ? v.z : v.w; };
            const uint32_t b0 = __byte_perm(word(vb[hf][0]), word(vb[hf][1]), sel), b1 = __byte_perm(word(vb[hf][2]), word(vb[hf][3]), sel);
            mma_bf16_m16n8k16(c, w[2 * hf][0], w[2 * hf][1], w[2 * hf + 1][0], w[2 * hf + 1][1], b0, b1);
            if (!FOLD) mma_bf16_m16n8k16(c, third[2 * hf], 0u, third[2 * hf + 1], 0u, b0, b1);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) o[8 * h + e][k] += c[k];
        }
      }
    } else {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)  // 16 slots per MMA
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          uint4 vb[4];
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int row = 16 * hf + 2 * tig + (s & 1) + 8 * (s >> 1);
            vb[s] = vr[h * GRP * 8 + row * 8 + (gid ^ (row & 7))];
          }
          const uint32_t w0[4] = {vb[0].x, vb[0].y, vb[0].z, vb[0].w};
          const uint32_t w1[4] = {vb[1].x, vb[1].y, vb[1].z, vb[1].w};
          const uint32_t w2[4] = {vb[2].x, vb[2].y, vb[2].z, vb[2].w};
          const uint32_t w3[4] = {vb[3].x, vb[3].y, vb[3].z, vb[3].w};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t sel = (e & 1) ? 0x7632u : 0x5410u;
            const uint32_t b0 = __byte_perm(w0[e >> 1], w1[e >> 1], sel);
            const uint32_t b1 = __byte_perm(w2[e >> 1], w3[e >> 1], sel);
            mma_bf16_m16n8k16(o[8 * h + e], w[2 * hf][0], w[2 * hf][1], w[2 * hf + 1][0], w[2 * hf + 1][1], b0, b1);
          }
        }
    }
  }
  if (!ok) {  // gave up on a copy: count it, and let what is in flight land (bounded) before the rings are reused
    if (lane == 0) {
      atomicAdd(&g_tc_error, 1);
      for (int b = 0; b < NBUF; ++b)
        for (uint32_t i = 0; i < kAttendSpinLimit; ++i) {
          uint32_t done;
          asm volatile(
              "{\n\t.reg .pred p;\n\t"
              "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
              "selp.u32 %0, 1, 0, p;\n\t}"
              : "=r"(done)
              : "r"(full(b)), "r"(b < buf ? phase : phase ^ 1u)
              : "memory");
          if (done) break;
        }
    }
    __syncwarp();
  }
  __syncthreads();  // the rings give way to the partial results
  // Per-warp partial result. l is summed over the quad (m and corr were equal across it).
  l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
  l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
  if (FOLD) {  // the third terms' share
#pragma unroll
    for (int t = 0; t < 8 * NH; ++t)
#pragma unroll
      for (int k = 0; k < 2; ++k) o[t][k] += __shfl_down_sync(0xFFFFFFFFu, o[t][k], 16);
  }
  if (gid < G) {
    if (tig == 0) part_ml[(warp * G + gid) * 2] = m, part_ml[(warp * G + gid) * 2 + 1] = l;
#pragma unroll
    for (int t = 0; t < 8 * NH; ++t) {
      const int h = t >> 3, e = t & 7;
      const int c0 = (2 * tig + 8 * h) * 8 + e, c1 = c0 + 8;
      if (!BELOW || c0 < d) part_o[(warp * G + gid) * d + c0] = o[t][0] + o[t][2];
      if (!BELOW || c1 < d) part_o[(warp * G + gid) * d + c1] = o[t][1] + o[t][3];
    }
  }
  __syncthreads();
  if (S == 1) {
    attend_merge<NW>(part_ml, part_o, G, d, a.out + (size_t)unit * G * d);
    return;
  }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  attend_merge_cluster<NW>(part_ml, part_o, gather, bar, G, d, S, rank, a.out + (size_t)unit * G * d);
}

// ------------------------------------------------------------------------------------------------ he_attend_scored, any dtype and d
//
// 64 slots at a time in shared memory as fp32, K rows padded so that lanes that read neighbouring rows meet every bank once. Scores: a warp
// works for one query head (8 / GP warps share a head's slots, GP the group rounded up to a power of two), a lane for one or more slots.
// Output: warp w adds up slots 8 w .. 8 w + 7 of the tile for all heads, a lane for four channels of every 128. A cluster of S CTAs shares a
// unit as in attend_bf16_kernel. Bound by the bytes in flight: a tile of 64 KB a CTA at most, with the scores and the output of the tile before in between.
// Measured, fp32 at d = 128: 8 units of 4096 slots 29 us (188 us with one CTA a unit; HBM needs 5.2), 128 units of 1024 slots 47 us, 2.9 TB/s (55 us with one
// CTA a unit; HBM needs 21); bf16 at d = 256, whose rows go through registers: 52 and 105 us;
// 4 units of 64 slots at d = 64 4.3 us, the latency of a launch and of two dependent reads.
// Hidden slots are not read at all: their rows are zeros. fp32 rows are copied asynchronously, with `stages` = 2 a tile ahead (calls that leave an SM
// to one CTA); which slots of a tile are hidden is found out one tile earlier still, so that no copy waits for a position (28 us, 31 with one stage).
constexpr int kScoredSlots = 64;
inline size_t scored_smem(int S, int stages, int G, int d) {
  const size_t tiles = (size_t)stages * kScoredSlots * (2 * d + 4), merge = (size_t)8 * G * (d + 2);
  return sizeof(float) * ((size_t)G * d + (tiles > merge ? tiles : merge) + kScoredSlots * 8 + 64 + (S > 1 ? (size_t)S * G * (d + 2) : 0));
}
// 16 bytes into shared memory, or zeros
__device__ __forceinline__ void cp_async16_or_zero(void* smem_dst, const void* gmem_src, bool some) {
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(smem_dst);
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(gmem_src), "r"(some ? 16u : 0u) : "memory");
}

template <int E, int GP>
__global__ void __launch_bounds__(kAttendThreads) attend_scored_kernel(const ScoredArgs a, const int S, const int stages) {
  extern __shared__ __align__(16) float asm_[];
  __shared__ __align__(8) unsigned long long merge_bar;
  const he_config& cfg = a.cfg;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int seq = a.n_order > 0 ? a.order[blockIdx.y] : blockIdx.y;
  const int rank = blockIdx.x % S, head = blockIdx.x / S, unit = seq * cfg.n_kv_heads + head;
  const int d = cfg.head_dim, G = cfg.group_size, pitch = d + 4;
  float* qs = asm_;                                  // [G][d]
  float* ks = qs + G * d;                            // [64][d + 4], then vs [64][d]; at the end part_ml, part_o
  const int stage_floats = kScoredSlots * (2 * d + 4), tiles_floats = stages * stage_floats, merge_floats = 8 * G * (d + 2);
  float* ps = ks + max(tiles_floats, merge_floats);  // [64 slots][8] weights
  float* stat = ps + kScoredSlots * 8;               // [8] factors of the output, then what warps tell each other (see below)
  uint32_t* seen_s = reinterpret_cast<uint32_t*>(stat + 32);  // [3][2] visible slots of a tile, by turns
  float* gather = stat + 64;
  const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&merge_bar);
  griddep_launch_dependents();
  if (S > 1) {
    if (rank == 0 && tid == 0) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)((S - 1) * G * (d + 2) * 4)) : "memory");
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // waited for before the first remote store
  }
  griddep_wait();
  const int fill = __ldcg(a.ca.fill + unit), now = __ldcg(a.ca.next_pos + unit) - 1;
  int low = a.mod.first_pos != nullptr ? max(0, a.mod.first_pos[seq]) : 0;
  if (a.mod.window > 0) low = max(low, now - a.mod.window + 1);
  const int cpr = d * E / 16;
  for (int i = tid; i < G * cpr; i += kAttendThreads) stage_chunk(qs + (i / cpr) * d, static_cast<const char*>(a.q) + ((size_t)unit * G + i / cpr) * d * E, i % cpr, cfg.dtype);
  const char* Kb = static_cast<const char*>(a.ca.k_cache) + (size_t)unit * cfg.max_budget * d * E;
  const char* Vb = static_cast<const char*>(a.ca.v_cache) + (size_t)unit * cfg.max_budget * d * E;
  const int32_t* pos = a.ca.pos + (size_t)unit * cfg.max_budget;
  constexpr int WPH = 8 / GP, MINE = kScoredSlots / (32 * WPH) > 0 ? kScoredSlots / (32 * WPH) : 1;  // warps of a head, slots of a lane
  constexpr int LANES = kScoredSlots / (WPH * MINE);                                                   // lanes of a warp with slots
  const int g = warp / WPH, part = warp % WPH;
  const float slope = a.mod.slopes != nullptr && g < G ? a.mod.slopes[head * G + g] * kLog2e : 0.f;
  float m = -INFINITY, l = 0.f;  // of head g; l of this lane's slots
  float o[8][8];                 // [head][channel 4 lane + e, 128 + 4 lane + e]
#pragma unroll
  for (int h = 0; h < 8; ++h)
#pragma unroll
    for (int e = 0; e < 8; ++e) o[h][e] = 0.f;
  const int step = kScoredSlots * S, j_first = kScoredSlots * rank;
  auto look = [&](int tile) {  // which slots of a tile are visible (warps 0 and 1)
    if (warp < 2) {
      const int j = j_first + tile * step + 32 * warp + lane;
      const uint32_t bits = __ballot_sync(0xFFFFFFFFu, j < fill && __ldcg(pos + j) >= low);
      if (lane == 0) seen_s[2 * (tile % 3) + warp] = bits;
    }
  };
  const int r_first = tid / cpr, c_first = tid % cpr, r_step = kAttendThreads / cpr, c_step = kAttendThreads % cpr;
  auto fetch = [&](int tile) {
    float* kt = ks + (stages == 2 ? tile & 1 : 0) * stage_floats;
    float* vt = kt + kScoredSlots * pitch;
    const int j0 = j_first + tile * step;
    const uint32_t seen[2] = {seen_s[2 * (tile % 3)], seen_s[2 * (tile % 3) + 1]};
    int r = r_first, c = c_first;
    auto next = [&]() {
      r += r_step, c += c_step;
      if (c >= cpr) c -= cpr, ++r;
    };
    auto visible = [&](int row) { return ((row < 32 ? seen[0] : seen[1]) >> (row & 31)) & 1u; };
    if (E == 4) {
      for (; r < kScoredSlots; next()) {
        const bool some = visible(r) != 0u;
        const size_t at = ((size_t)(some ? j0 + r : 0) * d) * E + 16 * c;
        cp_async16_or_zero(kt + r * pitch + 4 * c, Kb + at, some);
        cp_async16_or_zero(vt + r * d + 4 * c, Vb + at, some);
      }
    } else {
      while (r < kScoredSlots) {  // four rows' chunks at a time in registers
        uint4 k4[4], v4[4];
        int rr[4], cc[4];
#pragma unroll
        for (int u = 0; u < 4; ++u, next()) {
          rr[u] = r, cc[u] = c;
          k4[u] = v4[u] = make_uint4(0u, 0u, 0u, 0u);
          if (r < kScoredSlots && visible(r)) {
            const size_t at = ((size_t)(j0 + r) * d) * E + 16 * c;
            k4[u] = ldg_stream16(reinterpret_cast<const uint4*>(Kb + at)), v4[u] = ldg_stream16(reinterpret_cast<const uint4*>(Vb + at));
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (rr[u] < kScoredSlots) store_chunk(kt + rr[u] * pitch, k4[u], cc[u], HE_DTYPE_BF16), store_chunk(vt + rr[u] * d, v4[u], cc[u], HE_DTYPE_BF16);
      }
    }
    cp_async_commit();
  };
  const int tiles = j_first < fill ? (fill - j_first + step - 1) / step : 0;
  look(0), look(1);
  __syncthreads();
  if (tiles > 0) fetch(0);
  for (int tile = 0; tile < tiles; ++tile) {
    const int j0 = j_first + tile * step;
    const float* kt = ks + (stages == 2 ? tile & 1 : 0) * stage_floats;
    const float* vt = kt + kScoredSlots * pitch;
    look(tile + 2);
    if (stages == 2 && tile + 1 < tiles) {
      fetch(tile + 1);
      cp_async_wait_pending(1);
    } else {
      cp_async_wait_all();
    }
    int p[MINE];
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
      const int r = part * LANES * MINE + u * LANES + lane % LANES;
      p[u] = j0 + r < fill ? __ldcg(pos + j0 + r) : -1;
    }
    __syncthreads();
    // scores of head g
    float x[MINE], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
      const int r = part * LANES * MINE + u * LANES + lane % LANES;
      float s4[4] = {0.f, 0.f, 0.f, 0.f};
      if (g < G)
        for (int c = 0; c < d; c += 4) {
          const float4 k4 = *reinterpret_cast<const float4*>(kt + r * pitch + c), q4 = *reinterpret_cast<const float4*>(qs + g * d + c);
          s4[0] = fmaf(k4.x, q4.x, s4[0]), s4[1] = fmaf(k4.y, q4.y, s4[1]), s4[2] = fmaf(k4.z, q4.z, s4[2]), s4[3] = fmaf(k4.w, q4.w, s4[3]);
        }
      const float dot = (s4[0] + s4[1]) + (s4[2] + s4[3]);
      float y = a.mod.cap_log2 > 0.f ? a.mod.cap_log2 * tanhf(dot * a.mod.inv_cap) : dot * a.mod.scale_log2;
      y -= slope * (float)abs(now - p[u]);
      x[u] = p[u] >= low ? y : -INFINITY;
      top = fmaxf(top, x[u]);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
    if (WPH > 1) {  // a head's warps agree on the maximum
      if (lane == 0) stat[8 + warp] = top;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < WPH; ++u) top = fmaxf(top, stat[8 + g * WPH + u]);
    }
    const float mx = fmaxf(m, top), mn = mx == -INFINITY ? 0.f : mx, corr = exp2f(m - mn);
    m = mx;
    l *= corr;
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
      const int r = part * LANES * MINE + u * LANES + lane % LANES;
      const float w = exp2f(x[u] - mn);
      if (lane < LANES) l += w, ps[r * 8 + g] = w;
    }
    if (part == 0 && lane == 0) stat[g] = corr;
    __syncthreads();
    // output: this warp's slots
    float f[8];
    *reinterpret_cast<float4*>(f) = *reinterpret_cast<const float4*>(stat);
    if (GP > 4) *reinterpret_cast<float4*>(f + 4) = *reinterpret_cast<const float4*>(stat + 4);
#pragma unroll
    for (int h = 0; h < GP; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[h][e] *= f[h];
#pragma unroll 2
    for (int r = 8 * warp; r < 8 * warp + 8; ++r) {
      float w[8];
      *reinterpret_cast<float4*>(w) = *reinterpret_cast<const float4*>(ps + r * 8);
      if (GP > 4) *reinterpret_cast<float4*>(w + 4) = *reinterpret_cast<const float4*>(ps + r * 8 + 4);
#pragma unroll
      for (int part_c = 0; part_c < 2; ++part_c) {
        const int c = 128 * part_c + 4 * lane;
        if (c < d) {
          const float4 v4 = *reinterpret_cast<const float4*>(vt + r * d + c);
#pragma unroll
          for (int h = 0; h < GP; ++h) {
            o[h][4 * part_c] = fmaf(w[h], v4.x, o[h][4 * part_c]), o[h][4 * part_c + 1] = fmaf(w[h], v4.y, o[h][4 * part_c + 1]);
            o[h][4 * part_c + 2] = fmaf(w[h], v4.z, o[h][4 * part_c + 2]), o[h][4 * part_c + 3] = fmaf(w[h], v4.w, o[h][4 * part_c + 3]);
          }
        }
      }
    }
    __syncthreads();  // the tile has been read
    if (stages == 1 && tile + 1 < tiles) fetch(tile + 1);
  }
  __syncthreads();
  // every warp's share of the output, the sums by the warps that hold them
  float* part_ml = ks;
  float* part_o = ks + 8 * G * 2;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, off);
  if (lane == 0) stat[16 + warp] = m, stat[24 + warp] = l;
  __syncthreads();
  for (int h = lane; h < G; h += 32) {
    float lw = 0.f;  // (counted once: by warp 0)
    if (warp == 0)
      for (int u = 0; u < WPH; ++u) lw += stat[24 + h * WPH + u];
    part_ml[(warp * G + h) * 2] = stat[16 + h * WPH], part_ml[(warp * G + h) * 2 + 1] = lw;
  }
#pragma unroll
  for (int h = 0; h < GP; ++h)
    if (h < G)
#pragma unroll
      for (int part_c = 0; part_c < 2; ++part_c) {
        const int c = 128 * part_c + 4 * lane;
        if (c < d)
#pragma unroll
          for (int e = 0; e < 4; ++e) part_o[(warp * G + h) * d + c + e] = o[h][4 * part_c + e];
      }
  __syncthreads();
  if (S == 1) {
    attend_merge<8>(part_ml, part_o, G, d, a.out + (size_t)unit * G * d);
    return;
  }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  attend_merge_cluster<8>(part_ml, part_o, gather, bar, G, d, S, rank, a.out + (size_t)unit * G * d);
}

}  // namespace he
