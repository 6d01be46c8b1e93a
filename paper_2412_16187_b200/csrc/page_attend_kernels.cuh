// he_page_attend on the tensor cores: one token per sequence over pages of bf16 rows or of 8-bit codes, d <= 128, G <= 8.
//   out[g] = sum_j softmax_j(x_gj) V_j,  x_gj = cap / bias(scale q_g . K_j),  j in [low, len) of a sequence
// Bound by HBM: each visible row of K and V is read once for the group of query heads. What a call reads is known on the device alone (lengths, windows), and
// sequences may differ by any factor, so the work is dealt out there: all visible tokens of all sequences and KV heads ("units"), in groups of 32, form one line
// that is cut into as many equal parts as there are CTAs (one per SM, eight warps), each part into eight for its warps. A warp walks over its groups, whatever units
// they belong to, with an online softmax (running maximum, sum, unnormalised output in fp32); units that end within a warp are written at once, the pieces of others
// are put together in the CTA and, where a unit runs on into the next CTA, by page_join_kernel from a workspace. All sums have a fixed order.
//
// The rows come through rings of TMA tiles, 24 KB a warp, as in attend_bf16_kernel, whose register layout of the products this kernel shares: query heads
// are the rows of m16n8k16 MMAs, and the order of the channels in a product is chosen to suit 16-byte reads of the swizzled tiles.
//
// 8-bit codes go into the products as half precision, which holds every e4m3 value: one conversion instruction makes two. A page's scale multiplies its scores and its share
// of the output, so nothing is rounded on the way. Queries are scaled by a power of two per row to just below 2^14, where half precision holds all of a bf16 row but
// for what lies below 2^-38 of its largest entry; an fp32 row is two such terms, the second in MMA rows 8 to 15. Weights are
// taken times 2^14 (below 2^-38 of the largest they are lost) and split into two half-precision terms, the second again in rows 8 to 15: 2^-22 of each is left out.
// bf16 rows: as attend_bf16_kernel with MOD (three terms of a weight; rows 4..7 repeat heads 0..3 for the third ones up to G = 4). The products of a group start
// from zero and are added with rounding.
#pragma once
#include "attend_kernels.cuh"
#include "common.cuh"

namespace he {

constexpr int kPageGroup = 32;            // tokens of a group
template <bool Q8>
constexpr int kPageWarps = Q8 ? 12 : 8;
template <bool Q8>
constexpr int kPageRings = kPageWarps<Q8> * (Q8 ? 12 : 24) * 1024;  // bytes of a CTA's rings

struct PageMaps {
  alignas(64) CUtensorMap k, v;
};

template <int D, bool Q8>
struct PageRing {
  static constexpr int kRowBytes = Q8 ? D : 2 * D, kItemBytes = kPageGroup * kRowBytes, kBytes = kPageRings<Q8> / kPageWarps<Q8>, kBufs = kBytes / kItemBytes;
};
// Floats of a unit's piece: [G][d] outputs, [G] maxima in log2 units, [G] sums.
__host__ __device__ inline int page_piece(int G, int d) { return G * d + (2 * G + 3) / 4 * 4; }
template <bool Q8>
inline size_t page_attend_smem(int G, int d) { return 1024 + kPageRings<Q8> + kPageWarps<Q8> * page_piece(G, d) * sizeof(float); }
// What a CTA leaves for page_join_kernel: the unit whose first groups other CTAs have (-1: none), the unit whose last groups others have, then their pieces.
struct PageRest {
  int unit[2];
};
inline size_t page_workspace(int ctas, int G, int d) { return (size_t)ctas * (16 + 2 * (size_t)page_piece(G, d) * sizeof(float)); }
__device__ __forceinline__ PageRest* page_rest(float* part, int cta) { return reinterpret_cast<PageRest*>(part) + 2 * cta; }
__device__ __forceinline__ float* page_rest_piece(float* part, int ctas, int cta, int which, int piece) { return part + 4 * ctas + (2LL * cta + which) * piece; }

// The tokens [lo, hi) that the query of a sequence sees, and their groups [g0, g1).
struct PageSpan {
  int lo, hi, g0, g1;
};
static __device__ __noinline__ PageSpan page_span(const PagedAttendArgs& a, int s) {
  PageSpan p;
  p.hi = page_length(a.pages, s);
  p.lo = a.mod.first_pos != nullptr ? max(a.mod.first_pos[s], 0) : 0;
  if (a.mod.window > 0) p.lo = max(p.lo, p.hi - a.mod.window);
  p.lo = min(p.lo, p.hi);
  p.g0 = p.lo / kPageGroup, p.g1 = p.lo < p.hi ? (p.hi + kPageGroup - 1) / kPageGroup : p.g0;
  return p;
}

// A place on the line: group g of unit (s, h).
struct PageCursor {
  int s, h, g;
  PageSpan span;
};

// How the line of groups is cut: into `parts` of `each` groups, the first `more` parts one more, no fewer than a group per warp in each.
struct PageLine {
  long long each;
  int parts, more;
  __device__ __forceinline__ long long begin(int part) const { return part * each + min(part, more); }
};
// What the CTA's threads know of the sequences, `each` of them a thread (one, if there are not more sequences than threads): where its first one's groups begin on the line,
// and that sequence's span.
template <int THREADS>
struct PageTable {
  long long base[THREADS + 1];
  PageSpan span[THREADS];
};
template <int WARPS, typename F>
__device__ __forceinline__ PageLine page_line(const PagedAttendArgs& a, int ctas, int each, long long* scan_s, PageTable<32 * WARPS>& table, F empty) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  long long sum = 0;
#pragma unroll 1
  for (int i = 0, s = tid * each; i < each && s < a.cfg.batch; ++i, ++s) {
    const PageSpan p = page_span(a, s);
    sum += (p.g1 - p.g0) * a.cfg.n_kv_heads;
    if (i == 0) table.span[tid] = p;
    if (p.g1 == p.g0) empty(s);
  }
  long long incl = sum;
#pragma unroll
  for (int off = 1; off < 32; off *= 2) {
    const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, off);
    if (lane >= off) incl += up;
  }
  if (lane == 31) scan_s[warp] = incl;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w < warp) before += scan_s[w];
    total += scan_s[w];
  }
  table.base[tid] = before + incl - sum;
  if (tid == 0) table.base[32 * WARPS] = total;
  PageLine line;
  if (total >> 31 == 0) {  // (divisions of 32 bits are much the shorter ones)
    const unsigned n = (unsigned)total;
    line.parts = (int)max(1u, min((unsigned)ctas, (n + WARPS - 1) / WARPS));
    line.each = n / (unsigned)line.parts, line.more = (int)(n % (unsigned)line.parts);
  } else {
    line.parts = ctas, line.each = total / ctas, line.more = (int)(total % ctas);
  }
  __syncthreads();
  return line;
}
// Where group `at` of the line lies, by a whole warp: the last of the threads that begin no later, then that thread's sequences.
template <int WARPS>
__device__ __forceinline__ void page_find(const PagedAttendArgs& a, int each, const PageTable<32 * WARPS>& table, long long at, PageCursor& c) {
  const int lane = threadIdx.x & 31;
  const uint32_t coarse = __ballot_sync(0xFFFFFFFFu, lane < WARPS && table.base[32 * min(lane, WARPS - 1)] <= at);
  const int block = 31 - __clz(coarse);
  const int owner = 32 * block + 31 - __clz(__ballot_sync(0xFFFFFFFFu, table.base[32 * block + lane] <= at));
  // (threads behind the last one with groups begin at the end of the line, behind `at`; of several that begin at the same group, all but the last have none)
  c.s = owner * each, c.span = table.span[owner];
  int in = (int)(at - table.base[owner]);
  if (each > 1) {
#pragma unroll 1
    for (;;) {
      const int n = (c.span.g1 - c.span.g0) * a.cfg.n_kv_heads;
      if (in < n) break;
      in -= n, c.span = page_span(a, ++c.s);
    }
  }
  const int n = c.span.g1 - c.span.g0;
  c.h = in / n, c.g = c.span.g0 + in % n;
}

__device__ __forceinline__ float page_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma_f16_m16n8k16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_from_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16_from_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Pairs of fp32 values, two to an instruction.
__device__ __forceinline__ unsigned long long pair_of(float x, float y) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ unsigned long long pair_add(unsigned long long x, unsigned long long y) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}
__device__ __forceinline__ unsigned long long pair_fma(unsigned long long x, unsigned long long y, unsigned long long z) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
  return r;
}
__device__ __forceinline__ unsigned long long pair_mul(unsigned long long x, unsigned long long y) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}
__device__ __forceinline__ uint32_t half_pair(float x, float y) {  // x in the low half
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}
// x and y as a half-precision pair and what that leaves of them as another.
__device__ __forceinline__ void half_split(float x, float y, uint32_t& hi, uint32_t& lo) {
  hi = half_pair(x, y);
  const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  lo = half_pair(x - h.x, y - h.y);
}

// NBOX: pages of a group (2 for pages of 16 tokens). LO: the queries come in fp32 (8-bit pages). FOLD: G <= 4 (bf16 pages).
template <int D, bool Q8, int NBOX, bool LO, bool FOLD>
__global__ void __launch_bounds__(32 * kPageWarps<Q8>, 1) page_attend_kernel(const __grid_constant__ PagedAttendArgs a, float* part, const __grid_constant__ PageMaps maps) {
  using Ring = PageRing<D, Q8>;
  constexpr int WARPS = kPageWarps<Q8>, THREADS = 32 * WARPS, NBUF = Ring::kBufs, ITEM = Ring::kItemBytes, GRP = kPageGroup, NH = Q8 ? 1 : D / 64, SLOTS = (NBUF + 1) / 2;
  constexpr int NT = D / 8;  // output tiles of 8 channels
  extern __shared__ __align__(16) unsigned char page_smem_raw[];
  __shared__ __align__(8) unsigned long long ring_bar[WARPS][NBUF];
  __shared__ float scale_s[WARPS][SLOTS][4];  // of the groups under way: K's of each box, V's of each
  __shared__ int ent_unit[2 * WARPS], ent_flag[2 * WARPS];
  __shared__ long long scan_s[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const he_pages& pg = a.pages;
  const int H = a.cfg.n_kv_heads, G = a.cfg.group_size, d = a.cfg.head_dim, P = pg.page_size;
  unsigned char* smem = page_smem_raw + ((1024u - ((uint32_t)__cvta_generic_to_shared(page_smem_raw) & 1023u)) & 1023u);
  unsigned char* ring = smem + warp * Ring::kBytes;
  const int per = page_piece(G, d);
  // pieces of units that began before a warp's first group, and of those that go on behind its last one: in the place of its ring
  auto piece_of = [&](int e) { return reinterpret_cast<float*>((e & 1) ? smem + (e >> 1) * Ring::kBytes : smem + kPageRings<Q8> + (e >> 1) * per * sizeof(float)); };
  auto full = [&](int b) { return (uint32_t)__cvta_generic_to_shared(&ring_bar[warp][b]); };
  if (lane == 0) {
#pragma unroll
    for (int b = 0; b < NBUF; ++b) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(full(b)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    ent_unit[2 * warp] = ent_unit[2 * warp + 1] = -1;
  }
  griddep_wait();
  griddep_launch_dependents();
  // ---- the work: this CTA's part of the line, and where its warps begin
  PageTable<THREADS>& table = *reinterpret_cast<PageTable<THREADS>*>(smem);  // (the rings are not in use yet)
  static_assert(sizeof(PageTable<THREADS>) <= kPageRings<Q8>, "the rings hold the table");
  const int each = (a.cfg.batch + THREADS - 1) / THREADS;
  const PageLine line = page_line<WARPS>(a, gridDim.x, each, scan_s, table, [&](int s) {
    if (s % (int)gridDim.x == (int)blockIdx.x)
      for (int i = 0; i < H * G * d; i += 4) *reinterpret_cast<float4*>(a.out + (long long)s * H * G * d + i) = make_float4(0.f, 0.f, 0.f, 0.f);
  });
  PageRest* rest = page_rest(part, blockIdx.x);
  if (tid == 0) rest->unit[0] = rest->unit[1] = -1;
  if ((int)blockIdx.x >= line.parts) return;
  const long long begin = line.begin(blockIdx.x);
  const int some = (int)(line.begin(blockIdx.x + 1) - begin);  // groups of this CTA
  auto warp_begin = [&](int w) { return w * (some / WARPS) + min(w, some % WARPS); };
  const int groups = warp_begin(warp + 1) - warp_begin(warp), items = 2 * groups;
  PageCursor cur{}, ask{};  // the group that is worked on, the one that is asked for next
  if (groups > 0) page_find<WARPS>(a, each, table, begin + warp_begin(warp), cur);
  ask = cur;
  __syncthreads();  // the table has been read
  auto advance = [&](PageCursor& c) {
    if (++c.g < c.span.g1) return;
    if (++c.h == H) {
      c.h = 0;
#pragma unroll 1
      do c.span = page_span(a, ++c.s);
      while (c.span.g0 == c.span.g1);  // (there is another group)
    }
    c.g = c.span.g0;
  };
  // ---- copies. Lane i holds the page of box i & 1 of the group to be asked for, -1 where there is none, and fetches one of its scales.
  int page = -1;
  float scale = 0.f;
  auto look_up = [&]() {
    const int j = ask.g * GRP + (NBOX == 2 ? 16 * (lane & 1) : 0);
    page = j < ask.span.hi ? page_of(pg, ask.s, j) : -1;
  };
  if (groups > 0) look_up();
  const int none = pg.n_pages * H * P;  // a row behind all: zeros
  int row[NBOX], ask_slot = 0;
  // K (even t) or V of the next group into buffer b
  auto issue = [&](int t, int b) {
    const bool v = t & 1;
    if (Q8 && !v && t > 0 && t <= items) {  // the scales of the group before have come
      if (lane < 4) scale_s[warp][ask_slot][lane] = scale;
      if (++ask_slot == SLOTS) ask_slot = 0;
    }
    if (t >= items) return;
    if (!v) {
#pragma unroll
      for (int i = 0; i < NBOX; ++i) {
        const int p = NBOX == 2 ? __shfl_sync(0xFFFFFFFFu, page, i) : page;
        row[i] = p < 0 ? none : (p * H + ask.h) * P + ((ask.g * GRP + 16 * i) & (P - 1));
      }
      if (Q8) scale = lane < 4 && page >= 0 ? __ldcg((lane < 2 ? pg.k_scale : pg.v_scale) + (long long)page * H + ask.h) : 0.f;
    }
    if (lane == 0) {
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(ring + b * ITEM);
      const uint64_t map = v ? reinterpret_cast<uint64_t>(&maps.v) : reinterpret_cast<uint64_t>(&maps.k);
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full(b)), "r"((uint32_t)ITEM) : "memory");
#pragma unroll
      for (int i = 0; i < NBOX; ++i)
#pragma unroll
        for (int h = 0; h < NH; ++h)
          asm volatile(
              "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                  dst + h * GRP * 128 + i * (GRP / NBOX) * (Ring::kRowBytes / NH)),
              "l"(map), "r"(h * 64), "r"(row[i]), "r"(full(b))
              : "memory");
    }
    if (v && t + 1 < items) {
      advance(ask);
      look_up();
    }
  };
#pragma unroll 1
  for (int t = 0; t < NBUF - 1; ++t) issue(t, t);

  // ---- the queries of a unit
  const int my_head = !Q8 && FOLD ? gid & 3 : gid;
  constexpr int NQ = Q8 ? D / 64 * 8 : D / 32 * 4;
  uint32_t qf[NQ], ql[LO ? NQ : 1];
  float factor = a.mod.scale_log2, inv_cap = a.mod.inv_cap, slope = 0.f;
  auto load_q = [&]() {
    const long long at = (((long long)cur.s * H + cur.h) * G + my_head) * d;
    slope = a.mod.slopes != nullptr && my_head < G ? a.mod.slopes[cur.h * G + my_head] * kLog2e : 0.f;
    if constexpr (!Q8) {
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        uint4 t = make_uint4(0u, 0u, 0u, 0u);
        const int chunk = 2 * tig + (c & 1) + 8 * (c >> 1);
        if (my_head < G && chunk < d / 8) t = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.q) + 2 * (at + 8 * chunk));
        qf[4 * c] = t.x, qf[4 * c + 1] = t.y, qf[4 * c + 2] = t.z, qf[4 * c + 3] = t.w;
      }
    } else {
      float f[NQ * 2];
      uint32_t top = 0u;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const int c0 = 16 * (D == 128 ? 2 * tig + c : tig);  // (d is a multiple of 16)
#pragma unroll
        for (int e = 0; e < 16; e += LO ? 4 : 8) {
          uint4 t = make_uint4(0u, 0u, 0u, 0u);
          if (my_head < G && c0 < d) t = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.q) + (at + c0 + e) * (LO ? 4 : 2));
          const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
          for (int i = 0; i < (LO ? 4 : 8); ++i)
            f[16 * c + e + i] = LO ? __uint_as_float(w[i % 4]) : __uint_as_float((i & 1) ? w[(i / 2) % 4] & 0xFFFF0000u : w[(i / 2) % 4] << 16);
        }
      }
#pragma unroll
      for (int i = 0; i < NQ * 2; ++i) {
        const uint32_t bits = __float_as_uint(f[i]) & 0x7FFFFFFFu;
        top = max(top, bits < 0x7F800000u ? bits : 0u);
      }
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const int k = top == 0u ? 0 : min(13 - ((int)(top >> 23) - 127), 126);  // the row times 2^k is below 2^14
      const float up = __int_as_float((k + 127) << 23), down = __int_as_float((127 - k) << 23);
      factor = a.mod.scale_log2 * down, inv_cap = a.mod.inv_cap * down;
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        if constexpr (LO) half_split(f[2 * i] * up, f[2 * i + 1] * up, qf[i], ql[i]);
        else qf[i] = half_pair(f[2 * i] * up, f[2 * i + 1] * up);
      }
    }
  };
  // Outputs of columns 2 tig, 2 tig + 1 of each tile as pairs; bf16: of rows gid, then of rows gid + 8.
  constexpr int OW = Q8 ? 1 : 2;
  float m = -INFINITY, l = 0.f;
  unsigned long long o[NT][OW];
  auto clear = [&]() {
    m = -INFINITY, l = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < OW; ++e) o[t][e] = 0ull;
  };
  clear();
  int buf = 0, slot = 0;
  uint32_t phase = 0;
  bool ok = true, fresh = true, begins = false;
  // the next item has landed; its predecessor's buffer, read by the whole warp, takes the item NBUF - 1 ahead
  auto step = [&](int t) -> const unsigned char* {
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
    const unsigned char* p = ring + buf * ITEM;
    if (++buf == NBUF) buf = 0, phase ^= 1u;
    return p;
  };
  // where chunk c of row r of an 8-bit tile lies
  auto code_at = [&](const unsigned char* tile, int r, int c) { return tile + r * D + 16 * (D == 128 ? c ^ (r & 7) : c ^ ((r >> 1) & 3)); };
#pragma unroll 1
  for (int t = 0; t < items && ok; t += 2) {
    if (fresh) load_q(), begins = cur.g == cur.span.g0, fresh = false;
    const int j0 = cur.g * GRP, lo = cur.span.lo, hi = cur.span.hi;
    float sa[4][4], sb[4][4];
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    {
      const unsigned char* tile = step(t);
      if constexpr (Q8) {
        __syncwarp();
#pragma unroll
        for (int b = 0; b < NBOX; ++b) ks[b] = scale_s[warp][slot][b], vs[b] = scale_s[warp][slot][2 + b];
        if (++slot == SLOTS) slot = 0;
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 kv = *reinterpret_cast<const uint4*>(code_at(tile, 8 * i + gid, D == 128 ? 2 * tig + c : tig));
            const uint32_t w[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const uint32_t a0 = qf[8 * c + 2 * u], a1 = LO ? ql[LO ? 8 * c + 2 * u : 0] : 0u, a2 = qf[8 * c + 2 * u + 1], a3 = LO ? ql[LO ? 8 * c + 2 * u + 1 : 0] : 0u;
              const uint32_t b0 = e4m3_halves(w[u] & 0xFFFFu), b1 = e4m3_halves(w[u] >> 16);
              if (c == 0 && u == 0) mma_f16_from_zero(sa[i], a0, a1, a2, a3, b0, b1);
              else mma_f16_m16n8k16(sa[i], a0, a1, a2, a3, b0, b1);
            }
          }
      } else {
        const uint4* kr = reinterpret_cast<const uint4*>(tile) + gid * 8;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 kv = kr[(c >> 1) * GRP * 8 + i * 64 + ((2 * tig + (c & 1)) ^ gid)];
            if (c == 0) mma_bf16_from_zero(sa[i], qf[0], 0u, qf[1], 0u, kv.x, kv.y), mma_bf16_from_zero(sb[i], qf[2], 0u, qf[3], 0u, kv.z, kv.w);
            else mma_bf16_m16n8k16(sa[i], qf[4 * c], 0u, qf[4 * c + 1], 0u, kv.x, kv.y), mma_bf16_m16n8k16(sb[i], qf[4 * c + 2], 0u, qf[4 * c + 3], 0u, kv.z, kv.w);
          }
      }
    }
    // This lane: head gid, tokens j0 + 8 i + 2 tig, + 1.
    const bool edge = lo > j0 || hi < j0 + GRP;
    const uint32_t seen = (lo > j0 ? 0xFFFFFFFFu << (lo - j0) : 0xFFFFFFFFu) & (hi < j0 + GRP ? (1u << (hi - j0)) - 1u : 0xFFFFFFFFu);
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) x[2 * i + e] = Q8 ? (LO ? sa[i][e] + sa[i][2 + e] : sa[i][e]) : sa[i][e] + sb[i][e];
    if (a.mod.cap_log2 > 0.f) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = a.mod.cap_log2 * tanhf(x[k] * (inv_cap * ks[NBOX == 2 ? k >> 2 : 0]));
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= factor * ks[NBOX == 2 ? k >> 2 : 0];
    }
    if (a.mod.slopes != nullptr) {
      const float away = (float)(hi - 1 - j0 - 2 * tig);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = fmaf(-slope, away - (float)(8 * (k >> 1) + (k & 1)), x[k]);
    }
    if (edge) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = (seen >> (8 * (k >> 1) + 2 * tig + (k & 1))) & 1u ? x[k] : -INFINITY;
    }
    float gm = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 1));
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 2));
    constexpr float kUp = Q8 ? 14.f : 0.f;  // weights times 2^14: sums and outputs alike
    const float mx = fmaxf(m, gm), mn = mx == -INFINITY ? 0.f : mx;
    const float corr = page_ex2(m - mn);
    float p[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = page_ex2(x[k] - mn + kUp);
    l = l * corr + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
    m = mx;
    uint32_t w[4][2], third[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (Q8) {
        half_split(p[2 * i], p[2 * i + 1], w[i][0], w[i][1]);
      } else {
        split_pair(p[2 * i], p[2 * i + 1], w[i][0], w[i][1]);
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n"
            : "=r"(third[i])
            : "f"(p[2 * i + 1] - __uint_as_float(w[i][0] & 0xFFFF0000u) - __uint_as_float(w[i][1] & 0xFFFF0000u)),
              "f"(p[2 * i] - __uint_as_float(w[i][0] << 16) - __uint_as_float(w[i][1] << 16)));
        if (FOLD && gid >= 4) w[i][0] = third[i], w[i][1] = 0u;
      }
    }
    if (__any_sync(0xFFFFFFFFu, corr != 1.f)) {
      const unsigned long long both = pair_of(corr, corr);
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int e = 0; e < OW; ++e) o[u][e] = pair_mul(o[u][e], both);
    }
    const unsigned char* tile = step(t + 1);
    if constexpr (Q8) {
#pragma unroll
      for (int b = 0; b < NBOX; ++b)
        if (NBOX == 2 && ((seen >> (16 * b)) & 0xFFFFu) == 0u) vs[b] = 0.f;  // (a page that is not seen has any scale)
      unsigned long long scales[NBOX];
#pragma unroll
      for (int b = 0; b < NBOX; ++b) scales[b] = pair_of(vs[b], vs[b]);
#pragma unroll
      for (int q = 0; q < D / 64; ++q) {  // eight channels of each lane column at a time: tiles 8 q .. 8 q + 7
        uint2 v[2][4];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int r = 16 * hf + 2 * tig + (s & 1) + 8 * (s >> 1);
            v[hf][s] = *reinterpret_cast<const uint2*>(D == 128 ? code_at(tile, r, gid) + 8 * q : code_at(tile, r, gid >> 1) + 8 * (gid & 1));
            if (edge) {  // hidden rows (weighted by zero) hold anything: zeros
              const uint32_t keep = 0u - ((seen >> r) & 1u);
              v[hf][s].x &= keep, v[hf][s].y &= keep;
            }
          }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float c[NBOX][4][4];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            auto word = [&](int s) { return half ? v[hf][s].y : v[hf][s].x; };
            // codes of two tokens by channel
            const uint32_t a01 = __byte_perm(word(0), word(1), 0x5140u), a23 = __byte_perm(word(0), word(1), 0x7362u);
            const uint32_t b01 = __byte_perm(word(2), word(3), 0x5140u), b23 = __byte_perm(word(2), word(3), 0x7362u);
            const int set = NBOX == 2 ? hf : 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t first = e < 2 ? a01 : a23, second = e < 2 ? b01 : b23;
              const uint32_t b0 = e4m3_halves((e & 1) ? first >> 16 : first & 0xFFFFu), b1 = e4m3_halves((e & 1) ? second >> 16 : second & 0xFFFFu);
              if (NBOX == 2 || hf == 0) mma_f16_from_zero(c[set][e], w[2 * hf][0], w[2 * hf][1], w[2 * hf + 1][0], w[2 * hf + 1][1], b0, b1);
              else mma_f16_m16n8k16(c[set][e], w[2 * hf][0], w[2 * hf][1], w[2 * hf + 1][0], w[2 * hf + 1][1], b0, b1);
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int b = 0; b < NBOX; ++b) {
              unsigned long long& to = o[8 * q + 4 * half + e][0];
              to = pair_fma(pair_add(pair_of(c[b][e][0], c[b][e][1]), pair_of(c[b][e][2], c[b][e][3])), scales[b], to);
            }
        }
      }
    } else {
      const uint4* vr = reinterpret_cast<const uint4*>(tile);
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        uint4 vb[2][4];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int r = 16 * hf + 2 * tig + (s & 1) + 8 * (s >> 1);
            vb[hf][s] = vr[h * GRP * 8 + r * 8 + (gid ^ (r & 7))];
          }
        if (edge) {
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
          float c[4];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const uint32_t sel = (e & 1) ? 0x7632u : 0x5410u;
            auto word = [&](const uint4& v) { return (e >> 1) == 0 ? v.x : (e >> 1) == 1 ? v.y : (e >> 1) == 2 ? v.z : v.w; };
            const uint32_t b0 = __byte_perm(word(vb[hf][0]), word(vb[hf][1]), sel), b1 = __byte_perm(word(vb[hf][2]), word(vb[hf][3]), sel);
            if (hf == 0) mma_bf16_from_zero(c, w[0][0], w[0][1], w[1][0], w[1][1], b0, b1);
            else mma_bf16_m16n8k16(c, w[2][0], w[2][1], w[3][0], w[3][1], b0, b1);
            if (!FOLD) mma_bf16_m16n8k16(c, third[2 * hf], 0u, third[2 * hf + 1], 0u, b0, b1);
          }
          o[8 * h + e][0] = pair_add(o[8 * h + e][0], pair_of(c[0], c[1]));
          o[8 * h + e][OW - 1] = pair_add(o[8 * h + e][OW - 1], pair_of(c[2], c[3]));
        }
      }
    }
    const bool ends = cur.g + 1 == cur.span.g1;
    if (ends || t + 2 == items) {  // the unit's result, or this warp's piece of it
      l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
      l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
      const bool whole = begins && ends;
      const int e = 2 * warp + (ends ? 0 : 1);
      float* dst = whole ? a.out + ((long long)cur.s * H + cur.h) * G * d : piece_of(e);
      const float inv = whole ? (l != 0.f ? 1.f / l : 0.f) : 1.f;
      __syncwarp();  // (the ring has been read: its first bytes take the last piece)
#pragma unroll
      for (int u = 0; u < NT; u += 4) {
        float f[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          unsigned long long r = o[u + i][0];
          asm("mov.b64 {%0, %1}, %2;" : "=f"(f[0][i]), "=f"(f[1][i]) : "l"(r));
          if constexpr (!Q8) {
            if (FOLD) f[0][i] += __shfl_down_sync(0xFFFFFFFFu, f[0][i], 16), f[1][i] += __shfl_down_sync(0xFFFFFFFFu, f[1][i], 16);  // the third terms' share
            float f0, f1;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(f0), "=f"(f1) : "l"(o[u + i][OW - 1]));
            f[0][i] += f0, f[1][i] += f1;
          }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int n = 2 * tig + k;  // lane column: 8 bits: channels n * D / 8 + u; bf16: channels (n + 8 h) * 8 + e of tile 8 h + e
          const int ch = Q8 ? n * NT + u : (n + 8 * (u >> 3)) * 8 + (u & 7);
          if (gid < G && ch < d) *reinterpret_cast<float4*>(dst + gid * d + ch) = make_float4(f[k][0] * inv, f[k][1] * inv, f[k][2] * inv, f[k][3] * inv);
        }
      }
      if (!whole) {
        if (gid < G && tig == 0) dst[G * d + gid] = m, dst[G * d + G + gid] = l;
        if (lane == 0) ent_unit[e] = cur.s * H + cur.h, ent_flag[e] = (begins ? 1 : 0) | (ends ? 2 : 0);
      }
      clear();
      fresh = true;
    }
    if (t + 2 < items) advance(cur);
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
  __syncthreads();
  // ---- units that several warps share. Lane e has piece e; units are dealt out to the warps, several warps to one where there are few.
  const int mine = lane < 2 * WARPS ? ent_unit[lane] : -1;
  const uint32_t valid = __ballot_sync(0xFFFFFFFFu, mine >= 0), alike = __match_any_sync(0xFFFFFFFFu, mine);
  uint32_t leaders = __ballot_sync(0xFFFFFFFFu, mine >= 0 && lane == __ffs(alike) - 1);
  const int units = __popc(leaders);
  float* fold_s = reinterpret_cast<float*>(smem + warp * Ring::kBytes + 8192);  // [2 WARPS][8] weights of the pieces, behind this warp's own piece
  static_assert(kMaxGroup * (D + 2) * sizeof(float) <= 8192 && 8192 + 2 * WARPS * kMaxGroup * sizeof(float) <= Ring::kBytes && 2 * WARPS <= 32, "a ring holds its piece and the weights");
#pragma unroll 1
  for (int k = 0; leaders != 0u; ++k, leaders &= leaders - 1u) {
    if (units >= WARPS ? k % WARPS != warp : warp % units != k) continue;
    const int helpers = units >= WARPS ? 1 : (WARPS - 1 - k) / units + 1, helper = units >= WARPS ? 0 : warp / units;
    const int first = __ffs(leaders) - 1, unit = ent_unit[first];
    const uint32_t pieces = __ballot_sync(0xFFFFFFFFu, mine == unit) & valid;
    const int last = 31 - __clz(pieces);
    const bool from_start = ent_flag[first] & 1, whole = from_start && (ent_flag[last] & 2);
    const bool in = (pieces >> lane) & 1u;
    float* dst = whole ? a.out + (long long)unit * G * d : page_rest_piece(part, gridDim.x, blockIdx.x, from_start ? 1 : 0, per);
    float inv = 0.f;  // of head `lane`
#pragma unroll 1
    for (int g = 0; g < G; ++g) {
      const float mz = in ? piece_of(lane)[G * d + g] : -INFINITY;
      float M = mz;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, off));
      const float f = mz == -INFINITY ? 0.f : exp2f(mz - M);
      float L = in ? f * piece_of(lane)[G * d + G + g] : 0.f;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, off);
      if (in) fold_s[lane * kMaxGroup + g] = f;
      if (lane == g) inv = whole ? (L != 0.f ? 1.f / L : 0.f) : 1.f;
      if (!whole && helper == 0 && lane == 0) dst[G * d + g] = M, dst[G * d + G + g] = L;
    }
    __syncwarp();
#pragma unroll 1
    for (int at = helper * 32 + lane; at < (G * d / 4 + 31) / 32 * 32; at += 32 * helpers) {
      const int i = min(4 * at, G * d - 4), g = i / d;
      float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
      for (uint32_t rest_of = pieces; rest_of != 0u; rest_of &= rest_of - 1u) {
        const int z = __ffs(rest_of) - 1;
        const float4 v = *reinterpret_cast<const float4*>(piece_of(z) + i);
        const float f = fold_s[z * kMaxGroup + g];
        O.x = fmaf(v.x, f, O.x), O.y = fmaf(v.y, f, O.y), O.z = fmaf(v.z, f, O.z), O.w = fmaf(v.w, f, O.w);
      }
      const float by = __shfl_sync(0xFFFFFFFFu, inv, g);
      if (4 * at < G * d) *reinterpret_cast<float4*>(dst + i) = make_float4(O.x * by, O.y * by, O.z * by, O.w * by);
    }
    __syncwarp();
    if (!whole && helper == 0 && lane == 0) rest->unit[from_start ? 1 : 0] = unit;
  }
}

// Units that several CTAs share: the CTA that has a unit's second part puts all of its pieces together, a thread for four channels, in one pass over the pieces with a
// running maximum. (Few registers and threads, so that it waits beside the kernel before it, and few loads that wait for others: what it takes is latency.)
constexpr int kPageJoinThreads = 128;
static __global__ void __launch_bounds__(kPageJoinThreads) page_join_kernel(float* part, float* out, int ctas, int G, int d) {
  __shared__ int last_s;
  const int c = blockIdx.x + 1, tid = threadIdx.x, per = page_piece(G, d);
  if (tid == 0) last_s = ctas;
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();
  const int unit = __ldcg(&page_rest(part, c)->unit[0]), before = __ldcg(&page_rest(part, c - 1)->unit[1]);
  for (int z = c + 1 + tid; z < ctas; z += kPageJoinThreads)
    if (__ldcg(&page_rest(part, z)->unit[0]) != unit) {
      atomicMin(&last_s, z);
      break;
    }
  if (unit < 0 || before != unit) return;
  __syncthreads();
  const int last = last_s;
  for (int i = 4 * tid; i < G * d; i += 4 * kPageJoinThreads) {
    const int g = i / d;
    float M = -INFINITY, L = 0.f;
    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 5
    for (int z = c - 1; z < last; ++z) {
      const float* p = page_rest_piece(part, ctas, z, z < c ? 1 : 0, per);
      const float mz = __ldcg(p + G * d + g), lz = __ldcg(p + G * d + G + g);
      const float4 oz = __ldcg(reinterpret_cast<const float4*>(p + i));
      const float top = fmaxf(M, mz), ref = top == -INFINITY ? 0.f : top, f = exp2f(M - ref), fz = exp2f(mz - ref);
      L = L * f + lz * fz;
      O.x = O.x * f + oz.x * fz, O.y = O.y * f + oz.y * fz, O.z = O.z * f + oz.z * fz, O.w = O.w * f + oz.w * fz;
      M = top;
    }
    const float inv = L != 0.f ? 1.f / L : 0.f;
    *reinterpret_cast<float4*>(out + (long long)unit * G * d + i) = make_float4(O.x * inv, O.y * inv, O.z * inv, O.w * inv);
  }
}

}  // namespace he
