// he_page_attend on the tensor cores: one token per sequence over pages of bf16 rows or of 8-bit codes, d <= 128, G <= 8.
//   out[g] = sum_j softmax_j(x_gj) V_j,  x_gj = cap / bias(scale q_g . K_j),  j in [low, len) of a sequence
// Bound by HBM: each visible row of K and V is read once for the group of query heads. What a call reads is known on the device alone (lengths, windows), and
// sequences may differ by any factor, so the work is dealt out there: all visible tokens of all sequences and KV heads ("units"), in groups of 32, form one line
// that is cut into as many equal parts as there are CTAs (one per SM), each part into as many as it has warps. A warp walks over its groups, whatever units
// they belong to, with an online softmax (running maximum, sum, unnormalised output in fp32); units that end within a warp are written at once, the pieces of others
// are put together in the CTA and, where a unit runs on into the next CTA, by page_join_kernel from a workspace. All sums have a fixed order.
//
// The rows come through rings of TMA tiles, three items (K or V of a group) a warp. bf16 rows: the register layout of the products and the three terms of a weight are those
// of attend_bf16_kernel with MOD: query heads are the rows of m16n8k16 MMAs, the order of the channels in a product is chosen to suit 16-byte reads of the swizzled tiles, rows
// 4..7 repeat heads 0..3 for the third terms up to G = 4, the products of a group start from zero and are added with rounding.
//
// 8-bit codes go into the products as half precision, which holds every e4m3 value: one conversion instruction makes two. Tokens (K) and channels (V) are the rows of the
// MMAs and query heads the columns, so that all four registers of an A fragment hold codes; with heads as rows half of them are empty, and filling them in took the compiler
// 55 moves a group, twice as many MMAs and 20 % of the time. The weights come out of the first product as rows of tokens and go into the second as columns of heads: movmatrix
// turns them. A page's scale multiplies its scores and its share of the output, so nothing is rounded on the way. Queries are scaled by a power of two per row to just
// below 2^14, where half precision holds all of a bf16 row but for what lies below 2^-38 of its largest entry; an fp32 row is two such terms, with products of their own. Weights
// are taken times 2^14 (below 2^-38 of the largest they are lost) and split into two half-precision terms, the second in the columns of heads 4..7 up to G = 4, else with
// products of its own: 2^-22 of each is left out.
//
// Measured, d = 128 and G = 4 (HBM's copy rate in brackets): 512 units of 512 to 4096 tokens in 8 bits 59 us (47), of 2304 with fp32 queries 70 (46), 8 units of 32768 22 us (10), 8 of
// 131072 53 us (41); 128 units of 1024 to 8192 tokens in bf16 with bias, a quarter hidden, 55 us (43); 128 rows of d = 64 over 1500 plain keys 15 us (5). A call spends 4 us before its
// first copy has landed (lengths, the line, page numbers, each a trip to L2), 2 in a CTA's way out and 4 in page_join_kernel; the loop between them reads 5.8 to 6.3 TB/s. It issues 640
// instructions a group of 8-bit codes on half of its slots (128 of them conversions), 250 of bf16 rows.
#pragma once
#include "attend_kernels.cuh"
#include "common.cuh"
#include "tc_common.cuh"

namespace he {

constexpr int kPageGroup = 32;            // tokens of a group
constexpr float kPageFactorMax = 3.4028234e38f;  // the largest fp32 number
// Warps of a CTA: as many as hold their state in registers (168 each with 12 of them, 128 with 16). The loop waits for its own instructions, so more warps are faster: codes of
// 128 channels took 82 us with 10 warps and 69 with 12 at 512 units of 2304 tokens, and 65 with 16, which spill, where 12 took 60; codes of 64 channels 73 with 12 and 65 with 16.
template <int D, bool Q8>
constexpr int kPageWarps = Q8 ? (D == 128 ? 12 : 16) : 8;
constexpr int kPageBufs = 3;  // tiles of a warp's ring: K and V of a group by turns
template <int D, bool Q8>
constexpr int kPageRings = kPageWarps<D, Q8> * kPageBufs * kPageGroup * (Q8 ? D : 2 * D);  // bytes of a CTA's rings

struct PageMaps {
  alignas(64) CUtensorMap k, v;
};

template <int D, bool Q8>
struct PageRing {
  static constexpr int kRowBytes = Q8 ? D : 2 * D, kItemBytes = kPageGroup * kRowBytes, kBytes = kPageBufs * kItemBytes;
};
// Floats of a unit's piece: [G][d] outputs, [G] maxima in log2 units, [G] sums.
__host__ __device__ inline int page_piece(int G, int d) { return G * d + (2 * G + 3) / 4 * 4; }
template <int D, bool Q8>
inline size_t page_attend_smem(int G, int d) { return 1024 + kPageRings<D, Q8> + kPageWarps<D, Q8> * page_piece(G, d) * sizeof(float); }
// What a CTA leaves for page_join_kernel: the unit whose first groups other CTAs have (-1: none), the unit whose last groups others have, then their pieces.
struct PageRest {
  int unit[2];
};
inline size_t page_workspace(int ctas, int G, int d) { return (size_t)ctas * (16 + 2 * (size_t)page_piece(G, d) * sizeof(float)); }
__device__ __forceinline__ PageRest* page_rest(float* part, int cta) { return reinterpret_cast<PageRest*>(part) + 2 * cta; }
__device__ __forceinline__ float* page_rest_piece(float* part, int ctas, int cta, int which, int piece) { return part + 4 * ctas + (2LL * cta + which) * piece; }

// The same kernel for few rows over plain keys and values (he_attend_cross: bf16, at most 8 rows for a KV head, all of which see the same keys): cfg.group_size counts the
// rows of a unit, row g * rows + i being row i of query head g of the group.
struct RowsOver {
  const int32_t *q_len, *kv_len, *q_pos;  // [B]; q_pos or null: rows see all keys
  long long qs[3], os[3];                 // element strides (sequence, head, row)
  void* out;                              // bf16
  int keys, rows;
};
struct TokenArgs : PagedAttendArgs {
  RowsOver over;  // read with ROWS only
};

// The tokens [lo, hi) that the query of a sequence sees, their groups [g0, g1), and where the query's own token is.
struct PageSpan {
  int lo, hi, g0, g1, at;
};
template <bool ROWS>
static __device__ __noinline__ PageSpan page_span(const TokenArgs& a, int s) {
  PageSpan p;
  if constexpr (ROWS) {
    p.hi = min(max(a.over.kv_len[s], 0), a.over.keys), p.at = p.hi - 1;
    if (a.over.q_pos != nullptr) p.at = min(max(a.over.q_pos[s], -(1 << 24)), 1 << 24), p.hi = min(p.hi, max(p.at + 1, 0));
    p.lo = a.mod.first_pos != nullptr ? max(a.mod.first_pos[s * a.over.rows], 0) : 0;
    if (max(a.over.q_len[s], 0) == 0) p.lo = p.hi;
  } else {
    p.hi = page_length(a.pages, s), p.at = p.hi - 1;
    p.lo = a.mod.first_pos != nullptr ? max(a.mod.first_pos[s], 0) : 0;
  }
  if (a.mod.window > 0) p.lo = max(p.lo, p.at - a.mod.window + 1);
  p.lo = min(p.lo, p.hi);
  p.g0 = p.lo / kPageGroup, p.g1 = p.lo < p.hi ? (p.hi + kPageGroup - 1) / kPageGroup : p.g0;
  return p;
}
// A place on the line: group g of unit (s, h).
struct PageCursor {
  int s, h, g;
  PageSpan span;
};
// Four channels of a result.
template <bool ROWS>
__device__ __forceinline__ void page_emit(const TokenArgs& a, int unit, int row, int ch, const float4& v) {
  const int H = a.cfg.n_kv_heads, G = a.cfg.group_size;
  if constexpr (ROWS) {
    const int s = unit / H, g = row / a.over.rows, i = row % a.over.rows;
    if (i >= a.over.q_len[s]) return;
    uint2 two;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(two.x) : "f"(v.y), "f"(v.x));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(two.y) : "f"(v.w), "f"(v.z));
    const long long at = s * a.over.os[0] + ((long long)(unit % H) * (G / a.over.rows) + g) * a.over.os[1] + i * a.over.os[2] + ch;
    *reinterpret_cast<uint2*>(static_cast<char*>(a.over.out) + 2 * at) = two;
  } else {
    *reinterpret_cast<float4*>(a.out + ((long long)unit * G + row) * a.cfg.head_dim + ch) = v;
  }
}

__device__ __forceinline__ float page_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Pieces of a unit put together: maximum in log2 units, sum of the weights, four channels of the output.
struct PageSum {
  float M = -INFINITY, L = 0.f;
  float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void add(float m, float l, const float4& o) {
    const float top = fmaxf(M, m), ref = top == -INFINITY ? 0.f : top, f = page_ex2(M - ref), g = page_ex2(m - ref);
    L = fmaf(l, g, L * f), M = top;
    O.x = fmaf(o.x, g, O.x * f), O.y = fmaf(o.y, g, O.y * f), O.z = fmaf(o.z, g, O.z * f), O.w = fmaf(o.w, g, O.w * f);
  }
  __device__ __forceinline__ float4 result() const {
    const float inv = L != 0.f ? 1.f / L : 0.f;
    return make_float4(O.x * inv, O.y * inv, O.z * inv, O.w * inv);
  }
};

// Zeros for the sequences that see nothing, dealt out to the CTAs, by all threads of one and behind its first copies: 64 sequences of 2304 tokens (8 x 4 heads of 128, 8 bits) take
// 56 us with one of them empty and 57 without. (Written by the thread that counts the sequence's tokens, ahead of the copies: 109 us, and 514 instead of 47 for 32 x 8 heads of 300.)
template <int THREADS, bool ROWS>
static __device__ __noinline__ void page_zeros(const TokenArgs& a) {
  const int rows = a.cfg.n_kv_heads * a.cfg.group_size, d = a.cfg.head_dim;
#pragma unroll 1
  for (int s = blockIdx.x; s < a.cfg.batch; s += gridDim.x) {
    const PageSpan p = page_span<ROWS>(a, s);
    if (p.g0 != p.g1) continue;
    if constexpr (ROWS) {
      if (a.over.q_len[s] <= 0) continue;  // no rows
    }
#pragma unroll 1
    for (int i = 4 * threadIdx.x; i < rows * d; i += 4 * THREADS) {
      const int row = i / d;
      page_emit<ROWS>(a, s * a.cfg.n_kv_heads + row / a.cfg.group_size, row % a.cfg.group_size, i - row * d, make_float4(0.f, 0.f, 0.f, 0.f));
    }
  }
}

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
template <int WARPS, bool ROWS>
__device__ __forceinline__ PageLine page_line(const TokenArgs& a, int ctas, int each, long long* scan_s, PageTable<32 * WARPS>& table, int* empty_s) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  long long sum = 0;
#pragma unroll 1
  for (int i = 0, s = tid * each; i < each && s < a.cfg.batch; ++i, ++s) {
    const PageSpan p = page_span<ROWS>(a, s);
    sum += (p.g1 - p.g0) * a.cfg.n_kv_heads;
    if (i == 0) table.span[tid] = p;
    if (p.g1 == p.g0 && s % ctas == (int)blockIdx.x) *empty_s = 1;
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
template <int WARPS, bool ROWS>
__device__ __forceinline__ void page_find(const TokenArgs& a, int each, const PageTable<32 * WARPS>& table, long long at, PageCursor& c) {
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
      in -= n, c.span = page_span<ROWS>(a, ++c.s);
    }
  }
  const int n = c.span.g1 - c.span.g0;
  c.h = in / n, c.g = c.span.g0 + in % n;
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
// Rows of 8 x 8 values of 16 bits become columns (lane 4 r + c holds values 2 c, 2 c + 1 of row r).
__device__ __forceinline__ uint32_t half_turned(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
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

// A group under way: its unit, how far the query's token lies behind the group's first, which of its tokens are seen, whether it is the unit's first (1), last (2).
struct PageNow {
  int unit, away;
  uint32_t seen;
  int flags;
};

// NBOX: pages of a group (2 for pages of 16 tokens). LO: the queries come in fp32 (8-bit pages). FOLD: G <= 4 (bf16 pages).
template <int D, bool Q8, int NBOX, bool LO, bool FOLD, bool ROWS>
__global__ void __launch_bounds__(32 * kPageWarps<D, Q8>, 1) page_attend_kernel(const __grid_constant__ TokenArgs a, float* part, const __grid_constant__ PageMaps maps) {
  using Ring = PageRing<D, Q8>;
  constexpr int WARPS = kPageWarps<D, Q8>, THREADS = 32 * WARPS, NBUF = kPageBufs, ITEM = Ring::kItemBytes, GRP = kPageGroup, NH = Q8 ? 1 : D / 64;
  extern __shared__ __align__(16) unsigned char page_smem_raw[];
  __shared__ __align__(8) unsigned long long ring_bar[WARPS][NBUF];
  __shared__ int ent_unit[2 * WARPS], ent_flag[2 * WARPS];
  __shared__ long long scan_s[WARPS];
  __shared__ int empty_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const he_pages& pg = a.pages;
  const int H = a.cfg.n_kv_heads, G = a.cfg.group_size, d = a.cfg.head_dim, P = pg.page_size;
  unsigned char* smem = page_smem_raw + ((1024u - ((uint32_t)__cvta_generic_to_shared(page_smem_raw) & 1023u)) & 1023u);
  unsigned char* ring = smem + warp * Ring::kBytes;
  const int per = page_piece(G, d);
  // pieces of units that began before a warp's first group, and of those that go on behind its last one: in the place of its ring
  auto piece_of = [&](int e) { return reinterpret_cast<float*>((e & 1) ? smem + (e >> 1) * Ring::kBytes : smem + kPageRings<D, Q8> + (e >> 1) * per * sizeof(float)); };
  auto full = [&](int b) { return (uint32_t)__cvta_generic_to_shared(&ring_bar[warp][b]); };
  if (lane == 0) {
#pragma unroll
    for (int b = 0; b < NBUF; ++b) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(full(b)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    ent_unit[2 * warp] = ent_unit[2 * warp + 1] = -1;
  }
  if (tid == 0) empty_s = 0;
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();
  // ---- the work: this CTA's part of the line, and where its warps begin
  PageTable<THREADS>& table = *reinterpret_cast<PageTable<THREADS>*>(smem);  // (the rings are not in use yet)
  static_assert(sizeof(PageTable<THREADS>) <= kPageRings<D, Q8> && kMaxGroup * (D + 2) * sizeof(float) <= Ring::kBytes, "the rings hold the table, a ring the last piece");
  const int each = (a.cfg.batch + THREADS - 1) / THREADS;
  const PageLine line = page_line<WARPS, ROWS>(a, gridDim.x, each, scan_s, table, &empty_s);
  const bool empty = empty_s != 0;  // whether there are sequences that see nothing and whose outputs this CTA writes
  PageRest* rest = page_rest(part, blockIdx.x);
  if (tid == 0) rest->unit[0] = rest->unit[1] = -1;
  if ((int)blockIdx.x >= line.parts) {
    if (empty) page_zeros<THREADS, ROWS>(a);
    return;
  }
  const long long begin = line.begin(blockIdx.x);
  const int some = (int)(line.begin(blockIdx.x + 1) - begin);  // groups of this CTA
  auto warp_begin = [&](int w) { return w * (some / WARPS) + min(w, some % WARPS); };
  const int groups = warp_begin(warp + 1) - warp_begin(warp), items = 2 * groups;
  PageCursor ask{};  // the group that is asked for next
  if (groups > 0) page_find<WARPS, ROWS>(a, each, table, begin + warp_begin(warp), ask);
  fence_proxy_async();  // the table has been read, and copies come into its place
  __syncthreads();
  auto advance = [&](PageCursor& c) {
    if (++c.g < c.span.g1) return;
    if (++c.h == H) {
      c.h = 0;
#pragma unroll 1
      do c.span = page_span<ROWS>(a, ++c.s);
      while (c.span.g0 == c.span.g1);  // (there is another group)
    }
    c.g = c.span.g0;
  };
  // ---- the queries of a unit
  const int my_head = FOLD ? gid & 3 : gid;
  constexpr int NQ = Q8 ? D / 64 * 8 : D / 32 * 4;
  uint32_t qf[NQ], ql[LO ? NQ : 1];
  float slope[2] = {0.f, 0.f}, by[2] = {1.f, 1.f};  // of this lane's heads; by (8 bits): what makes a score of a product, or what its cap's tanh takes
  uint4 raw[Q8 && LO ? D / 16 : D / 32];  // as they lie in memory
  auto ask_q = [&](int unit) {
    long long at = ((long long)unit * G + my_head) * d;
    if constexpr (ROWS) at = unit / H * a.over.qs[0] + ((long long)(unit % H) * (G / a.over.rows) + my_head / a.over.rows) * a.over.qs[1] + my_head % a.over.rows * a.over.qs[2];
    if (a.mod.slopes != nullptr) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int g = !Q8 ? my_head : FOLD ? (2 * tig + k) & 3 : 2 * tig + k;
        slope[k] = g < G ? a.mod.slopes[unit % H * G + g] * kLog2e : 0.f;
      }
    }
    constexpr int PER = LO ? 4 : 8, EACH = Q8 ? 16 / PER : 1;  // channels of 16 bytes, such pieces in a lane's 16 channels
#pragma unroll
    for (int c = 0; c < (int)(sizeof(raw) / sizeof(uint4)); ++c) {
      // 8 bits: 16 channels a lane and 64 (d is a multiple of 16); bf16: 8
      const int ch = Q8 ? 16 * (D == 128 ? 2 * tig + c / EACH : tig) + c % EACH * PER : 8 * (2 * tig + (c & 1) + 8 * (c >> 1));
      raw[c] = make_uint4(0u, 0u, 0u, 0u);
      if (my_head < G && ch < d) raw[c] = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.q) + (at + ch) * (LO ? 4 : 2));
    }
  };
  auto take_q = [&]() {
    if constexpr (!Q8) {
#pragma unroll
      for (int c = 0; c < D / 32; ++c) qf[4 * c] = raw[c].x, qf[4 * c + 1] = raw[c].y, qf[4 * c + 2] = raw[c].z, qf[4 * c + 3] = raw[c].w;
    } else {
      float f[NQ * 2];
      uint32_t top = 0u;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
#pragma unroll
        for (int e = 0; e < 16; e += LO ? 4 : 8) {
          const uint4 t = raw[(16 * c + e) / (LO ? 4 : 8)];
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
      const float mine = fminf((a.mod.cap_log2 > 0.f ? a.mod.inv_cap : a.mod.scale_log2) * down, kPageFactorMax);  // of head gid
#pragma unroll
      for (int k = 0; k < 2; ++k) by[k] = __shfl_sync(0xFFFFFFFFu, mine, 4 * (2 * tig + k));
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        if constexpr (LO) {
          half_split(f[2 * i] * up, f[2 * i + 1] * up, qf[i], ql[i]);
          if (fabsf(f[2 * i]) == INFINITY) ql[i] &= 0xFFFF0000u;  // (an infinity has no second term)
          if (fabsf(f[2 * i + 1]) == INFINITY) ql[i] &= 0xFFFFu;
        } else {
          qf[i] = half_pair(f[2 * i] * up, f[2 * i + 1] * up);
        }
      }
    }
  };
  if (groups > 0) ask_q(ask.s * H + ask.h);
  // ---- copies. Lane i holds the page of box i & 1 of the group to be asked for, -1 where there is none or nothing of it is seen, and fetches one of its scales.
  int page = -1;
  float scale = 0.f;
  auto look_up = [&]() {
    const int j = ask.g * GRP + (NBOX == 2 ? 16 * (lane & 1) : 0);
    if constexpr (!ROWS) page = j < ask.span.hi && (NBOX == 1 || j + 16 > ask.span.lo) ? page_of(pg, ask.s, j) : -1;
  };
  if (groups > 0) look_up();
  PageNow now{}, next{};  // the group that is worked on, the last one whose V has been asked for
  const int none = pg.n_pages * H * P;  // a row behind all: zeros
  int row[NBOX];
  // K (even t) or V of the next group into buffer b
  auto issue = [&](int t, int b) {
    const bool v = t & 1;
    if (t >= items) return;
    if (!v && !ROWS) {
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
          if constexpr (ROWS) tma_load_4d(dst + h * GRP * 128, v ? &maps.v : &maps.k, 64 * h, ask.g * GRP, ask.h, ask.s, full(b));
          else asm volatile(
              "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                  dst + h * GRP * 128 + i * (GRP / NBOX) * (Ring::kRowBytes / NH)),
              "l"(map), "r"(h * 64), "r"(row[i]), "r"(full(b))
              : "memory");
    }
    if (v) {
      const int j0 = ask.g * GRP, lo = ask.span.lo - j0, hi = ask.span.hi - j0;
      next.unit = ask.s * H + ask.h, next.away = ask.span.at - j0;
      next.seen = (lo > 0 ? 0xFFFFFFFFu << lo : 0xFFFFFFFFu) & (hi < GRP ? (1u << hi) - 1u : 0xFFFFFFFFu);
      next.flags = (ask.g == ask.span.g0 ? 1 : 0) | (ask.g + 1 == ask.span.g1 ? 2 : 0);
      if (t + 1 < items) {
        advance(ask);
        look_up();
      }
    }
  };
#pragma unroll 1
  for (int t = 0; t < NBUF - 1; ++t) issue(t, t);
  if (empty) page_zeros<THREADS, ROWS>(a);  // (while the copies are under way)

  // bf16: outputs of columns 2 tig, 2 tig + 1 of each tile of 8 channels as pairs, of rows (heads) gid, then of rows gid + 8. 8 bits: of heads 2 tig, 2 tig + 1 as pairs, of rows
  // (channels) gid, then gid + 8 of each tile of 16.
  constexpr int NO = Q8 ? D / 16 : D / 8, HEADS = Q8 ? 2 : 1;  // heads of a lane
  float m[HEADS], l[HEADS];
  unsigned long long o[NO][2];
  auto clear = [&]() {
#pragma unroll
    for (int k = 0; k < HEADS; ++k) m[k] = -INFINITY, l[k] = 0.f;
#pragma unroll
    for (int t = 0; t < NO; ++t) o[t][0] = o[t][1] = 0ull;
  };
  clear();
  int buf = 0;
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
  // Rows of V that are hidden (weighted by zero) hold anything: zeros.
  auto hide = [&](const unsigned char* tile) {
    for (int i = lane; i < GRP * Ring::kRowBytes / 16; i += 32) {
      const int r = Q8 ? i / (D / 16) : (i >> 3) % GRP;
      if (((now.seen >> r) & 1u) == 0u) *reinterpret_cast<uint4*>(const_cast<unsigned char*>(tile) + 16 * i) = make_uint4(0u, 0u, 0u, 0u);
    }
    fence_proxy_async();  // (the next copy into these rows comes after them)
    __syncwarp();
  };
#pragma unroll 1
  for (int t = 0; t < items && ok; t += 2) {
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    if constexpr (Q8) {  // (three items in a ring: the next group's have not been asked for yet)
      static_assert(NBUF == 3, "scales of one group at a time");
#pragma unroll
      for (int b = 0; b < NBOX; ++b) ks[b] = __shfl_sync(0xFFFFFFFFu, scale, b), vs[b] = __shfl_sync(0xFFFFFFFFu, scale, 2 + b);
    }
    const unsigned char* tile = step(t);  // (V of this group has been asked for by now, that of the next one not: that is another step)
    now = next;
    if (fresh) take_q(), begins = now.flags & 1, fresh = false;
    const bool edge = now.seen != 0xFFFFFFFFu;
    if constexpr (Q8) {
      // S = K q^T: tokens 16 u + gid (+ 8), heads 2 tig, + 1
      float x[2][2][2];
      {
        float c[2][4];
#pragma unroll
        for (int w = 0; w < D / 64; ++w)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int ch = D == 128 ? 2 * tig + w : tig;
            const uint4 k0 = *reinterpret_cast<const uint4*>(code_at(tile, 16 * u + gid, ch)), k1 = *reinterpret_cast<const uint4*>(code_at(tile, 16 * u + 8 + gid, ch));
            const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t a0 = e4m3_halves(w0[i] & 0xFFFFu), a1 = e4m3_halves(w1[i] & 0xFFFFu), a2 = e4m3_halves(w0[i] >> 16), a3 = e4m3_halves(w1[i] >> 16);
              if (w == 0 && i == 0) mma_f16_from_zero(c[u], a0, a1, a2, a3, qf[0], qf[1]);
              else mma_f16_m16n8k16(c[u], a0, a1, a2, a3, qf[8 * w + 2 * i], qf[8 * w + 2 * i + 1]);
              if constexpr (LO) mma_f16_m16n8k16(c[u], a0, a1, a2, a3, ql[8 * w + 2 * i], ql[8 * w + 2 * i + 1]);
            }
          }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int k = 0; k < 2; ++k) x[u][r][k] = c[u][2 * r + k];
      }
      // (what makes a score of a product is finite, so that a product of zero is a score of zero)
      if (a.mod.cap_log2 > 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i >> 2][(i >> 1) & 1][i & 1] = a.mod.cap_log2 * tanhf(x[i >> 2][(i >> 1) & 1][i & 1] * fminf(by[i & 1] * ks[NBOX == 2 ? i >> 2 : 0], kPageFactorMax));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i >> 2][(i >> 1) & 1][i & 1] *= fminf(by[i & 1] * ks[NBOX == 2 ? i >> 2 : 0], kPageFactorMax);
      }
      if (a.mod.slopes != nullptr) {
        const float away = (float)(now.away - gid);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i >> 2][(i >> 1) & 1][i & 1] = fmaf(-slope[i & 1], away - (float)(8 * (i >> 1)), x[i >> 2][(i >> 1) & 1][i & 1]);
      }
      if (edge) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i >> 2][(i >> 1) & 1][i & 1] = (now.seen >> (8 * (i >> 1) + gid)) & 1u ? x[i >> 2][(i >> 1) & 1][i & 1] : -INFINITY;
      }
      float corr[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float gm = fmaxf(fmaxf(x[0][0][k], x[0][1][k]), fmaxf(x[1][0][k], x[1][1][k]));
        gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 4));
        gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 8));
        gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 16));
        const float mx = fmaxf(m[k], gm), mn = mx == -INFINITY ? 0.f : mx;
        corr[k] = page_ex2(m[k] - mn);
        m[k] = mx;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i >> 1][i & 1][k] = page_ex2((x[i >> 1][i & 1][k] - mn) + 14.f);  // weights times 2^14: sums and outputs alike (mn - 14 would be rounded)
        l[k] = fmaf(l[k], corr[k], (x[0][0][k] + x[0][1][k]) + (x[1][0][k] + x[1][1][k]));
      }
      // the weights of 8 tokens by 8 heads at a time, turned round: rows of tokens become the products' columns of heads
      uint32_t p[2][2], rest_p[FOLD ? 1 : 2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          uint32_t hi, lo;
          half_split(x[u][r][0], x[u][r][1], hi, lo);
          p[u][r] = half_turned(FOLD && tig >= 2 ? lo : hi);
          if constexpr (!FOLD) rest_p[u][r] = half_turned(lo);
        }
      if (__any_sync(0xFFFFFFFFu, corr[0] != 1.f || corr[1] != 1.f)) {
        const unsigned long long both = pair_of(corr[0], corr[1]);
#pragma unroll
        for (int i = 0; i < NO; ++i) o[i][0] = pair_mul(o[i][0], both), o[i][1] = pair_mul(o[i][1], both);
      }
      tile = step(t + 1);
      if (edge) hide(tile);
      unsigned long long scales[NBOX];
#pragma unroll
      for (int b = 0; b < NBOX; ++b) scales[b] = pair_of(vs[b], vs[b]);
      // O^T += V^T P^T: rows gid, gid + 8 of tile i are channels gid * D / 8 + 2 i, + 1
#pragma unroll
      for (int q = 0; q < D / 64; ++q) {  // eight of the lane's channels
        uint2 v[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int r = 16 * u + 2 * tig + (s & 1) + 8 * (s >> 1);
            v[u][s] = *reinterpret_cast<const uint2*>(D == 128 ? code_at(tile, r, gid) + 8 * q : code_at(tile, r, gid >> 1) + 8 * (gid & 1));
          }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float c[NBOX][4];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            auto word = [&](int s) { return i < 2 ? v[u][s].x : v[u][s].y; };
            // codes of two tokens, of two channels
            const uint32_t first = __byte_perm(word(0), word(1), i & 1 ? 0x7362u : 0x5140u), second = __byte_perm(word(2), word(3), i & 1 ? 0x7362u : 0x5140u);
            const uint32_t a0 = e4m3_halves(first & 0xFFFFu), a1 = e4m3_halves(first >> 16), a2 = e4m3_halves(second & 0xFFFFu), a3 = e4m3_halves(second >> 16);
            const int set = NBOX == 2 ? u : 0;
            if (NBOX == 2 || u == 0) mma_f16_from_zero(c[set], a0, a1, a2, a3, p[u][0], p[u][1]);
            else mma_f16_m16n8k16(c[set], a0, a1, a2, a3, p[u][0], p[u][1]);
            if constexpr (!FOLD) mma_f16_m16n8k16(c[set], a0, a1, a2, a3, rest_p[u][0], rest_p[u][1]);
          }
#pragma unroll
          for (int b = 0; b < NBOX; ++b) {
            o[4 * q + i][0] = pair_fma(pair_of(c[b][0], c[b][1]), scales[b], o[4 * q + i][0]);
            o[4 * q + i][1] = pair_fma(pair_of(c[b][2], c[b][3]), scales[b], o[4 * q + i][1]);
          }
        }
      }
    } else {
      // S = q K^T: head gid, tokens 8 i + 2 tig, + 1
      float x[8];
      {
        float sa[4][4], sb[4][4];
        const uint4* kr = reinterpret_cast<const uint4*>(tile) + gid * 8;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 kv = kr[(c >> 1) * GRP * 8 + i * 64 + ((2 * tig + (c & 1)) ^ gid)];
            if (c == 0) mma_bf16_from_zero(sa[i], qf[0], 0u, qf[1], 0u, kv.x, kv.y), mma_bf16_from_zero(sb[i], qf[2], 0u, qf[3], 0u, kv.z, kv.w);
            else mma_bf16_m16n8k16(sa[i], qf[4 * c], 0u, qf[4 * c + 1], 0u, kv.x, kv.y), mma_bf16_m16n8k16(sb[i], qf[4 * c + 2], 0u, qf[4 * c + 3], 0u, kv.z, kv.w);
          }
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = sa[k >> 1][k & 1] + sb[k >> 1][k & 1];
      }
      if (a.mod.cap_log2 > 0.f) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = a.mod.cap_log2 * tanhf(x[k] * a.mod.inv_cap);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= a.mod.scale_log2;
      }
      if (a.mod.slopes != nullptr) {
        const float away = (float)(now.away - 2 * tig);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = fmaf(-slope[0], away - (float)(8 * (k >> 1) + (k & 1)), x[k]);
      }
      if (edge) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (now.seen >> (8 * (k >> 1) + 2 * tig + (k & 1))) & 1u ? x[k] : -INFINITY;
      }
      float gm = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 1));
      gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 2));
      const float mx = fmaxf(m[0], gm), mn = mx == -INFINITY ? 0.f : mx;
      const float corr = page_ex2(m[0] - mn);
      float p[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) p[k] = page_ex2(x[k] - mn);
      l[0] = l[0] * corr + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
      m[0] = mx;
      uint32_t w[4][2], third[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        split_pair(p[2 * i], p[2 * i + 1], w[i][0], w[i][1]);
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n"
            : "=r"(third[i])
            : "f"(p[2 * i + 1] - __uint_as_float(w[i][0] & 0xFFFF0000u) - __uint_as_float(w[i][1] & 0xFFFF0000u)),
              "f"(p[2 * i] - __uint_as_float(w[i][0] << 16) - __uint_as_float(w[i][1] << 16)));
        if (FOLD && gid >= 4) w[i][0] = third[i], w[i][1] = 0u;
      }
      if (__any_sync(0xFFFFFFFFu, corr != 1.f)) {
        const unsigned long long both = pair_of(corr, corr);
#pragma unroll
        for (int i = 0; i < NO; ++i) o[i][0] = pair_mul(o[i][0], both), o[i][1] = pair_mul(o[i][1], both);
      }
      tile = step(t + 1);
      if (edge) hide(tile);
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
          o[8 * h + e][1] = pair_add(o[8 * h + e][1], pair_of(c[2], c[3]));
        }
      }
    }
    const bool ends = now.flags & 2;
    if (ends || t + 2 == items) {  // the unit's result, or this warp's piece of it
#pragma unroll
      for (int k = 0; k < HEADS; ++k) {
        l[k] += __shfl_xor_sync(0xFFFFFFFFu, l[k], Q8 ? 4 : 1);
        l[k] += __shfl_xor_sync(0xFFFFFFFFu, l[k], Q8 ? 8 : 2);
        if (Q8) l[k] += __shfl_xor_sync(0xFFFFFFFFu, l[k], 16);
      }
      const bool whole = begins && ends;
      const int e = 2 * warp + (ends ? 0 : 1);
      float* dst = piece_of(e);
      auto put = [&](int row, int ch, const float4& v) {
        if (whole) page_emit<ROWS>(a, now.unit, row, ch, v);
        else *reinterpret_cast<float4*>(dst + row * d + ch) = v;
      };
      float inv[HEADS];
#pragma unroll
      for (int k = 0; k < HEADS; ++k) inv[k] = whole ? (l[k] != 0.f ? 1.f / l[k] : 0.f) : 1.f;
      __syncwarp();  // (the ring has been read: its first bytes take the last piece)
      if constexpr (Q8) {
        const int first = FOLD ? 2 * (tig & 1) : 2 * tig;
#pragma unroll
        for (int i = 0; i < NO; i += 2) {
          float f[2][4];  // four channels of each head
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            asm("mov.b64 {%0, %1}, %2;" : "=f"(f[0][c]), "=f"(f[1][c]) : "l"(o[i + (c >> 1)][c & 1]));
            if (FOLD) f[0][c] += __shfl_xor_sync(0xFFFFFFFFu, f[0][c], 2), f[1][c] += __shfl_xor_sync(0xFFFFFFFFu, f[1][c], 2);  // the second terms' share
          }
          const int ch = gid * (D / 8) + 2 * i;
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if ((!FOLD || tig < 2) && first + k < G && ch < d)
              put(first + k, ch, make_float4(f[k][0] * inv[k], f[k][1] * inv[k], f[k][2] * inv[k], f[k][3] * inv[k]));
        }
        if (!whole && gid == 0 && (!FOLD || tig < 2)) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (first + k < G) dst[G * d + first + k] = m[k], dst[G * d + G + first + k] = l[k];
        }
      } else {
#pragma unroll
        for (int i = 0; i < NO; i += 4) {
          float f[2][4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float f0, f1;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(f[0][c]), "=f"(f[1][c]) : "l"(o[i + c][0]));
            if (FOLD) f[0][c] += __shfl_down_sync(0xFFFFFFFFu, f[0][c], 16), f[1][c] += __shfl_down_sync(0xFFFFFFFFu, f[1][c], 16);  // the third terms' share
            asm("mov.b64 {%0, %1}, %2;" : "=f"(f0), "=f"(f1) : "l"(o[i + c][1]));
            f[0][c] += f0, f[1][c] += f1;
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int ch = (2 * tig + k + 8 * (i >> 3)) * 8 + (i & 7);  // tile 8 h + e of lane column n is channel (n + 8 h) * 8 + e
            if (gid < G && ch < d) put(gid, ch, make_float4(f[k][0] * inv[0], f[k][1] * inv[0], f[k][2] * inv[0], f[k][3] * inv[0]));
          }
        }
        if (!whole && gid < G && tig == 0) dst[G * d + gid] = m[0], dst[G * d + G + gid] = l[0];
      }
      if (!whole && lane == 0) ent_unit[e] = now.unit, ent_flag[e] = (begins ? 1 : 0) | (ends ? 2 : 0);
      clear();
      fresh = true;
      if (t + 2 < items) ask_q(next.unit);  // (its V has been asked for)
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
  __syncthreads();
  // ---- units that several warps share. Lane e has piece e; a thread has four channels of each unit. (Little code: it comes from L2, past what other CTAs still read, and
  // was waited for longer than executed when units were dealt out to warps: 2 to 8 us.)
  const int mine = lane < 2 * WARPS ? ent_unit[lane] : -1;
  const uint32_t alike = __match_any_sync(0xFFFFFFFFu, mine);
  uint32_t leaders = __ballot_sync(0xFFFFFFFFu, mine >= 0 && lane == __ffs(alike) - 1);
  static_assert(2 * WARPS <= 32 && 4 * THREADS >= kMaxGroup * D, "a lane for each piece, a thread for four channels");
  const int i = 4 * tid, g = i / d;
#pragma unroll 1
  for (; leaders != 0u; leaders &= leaders - 1u) {
    const int first = __ffs(leaders) - 1;
    const uint32_t pieces = __shfl_sync(0xFFFFFFFFu, alike, first);
    const int unit = ent_unit[first], which = ent_flag[first] & 1;
    const bool whole = which && (ent_flag[31 - __clz(pieces)] & 2);
    if (i < G * d) {
      PageSum sum;
#pragma unroll 1
      for (uint32_t left = pieces; left != 0u; left &= left - 1u) {
        const float* p = piece_of(__ffs(left) - 1);
        sum.add(p[G * d + g], p[G * d + G + g], *reinterpret_cast<const float4*>(p + i));
      }
      float* dst = page_rest_piece(part, gridDim.x, blockIdx.x, which, per);
      if (whole) {
        page_emit<ROWS>(a, unit, g, i - g * d, sum.result());
      } else {
        *reinterpret_cast<float4*>(dst + i) = sum.O;
        if (i == g * d) dst[G * d + g] = sum.M, dst[G * d + G + g] = sum.L;
        rest->unit[which] = unit;
      }
    }
  }
}

// Units that several CTAs share: the CTA that has a unit's second part puts all of its pieces together, a thread for four channels, the pieces dealt out to as many shares of
// the threads as there are. What it takes is latency: of two loads that wait for others, and of the pieces' own, four in flight.
constexpr int kPageJoinThreads = 512;
template <bool ROWS>
static __global__ void __launch_bounds__(kPageJoinThreads) page_join_kernel(const __grid_constant__ TokenArgs a, float* part, int ctas) {
  __shared__ int last_s;
  __shared__ PageSum share_s[kPageJoinThreads];
  const int G = a.cfg.group_size, d = a.cfg.head_dim, c = blockIdx.x + 1, tid = threadIdx.x, per = page_piece(G, d), columns = G * d / 4, shares = kPageJoinThreads / columns;  // (columns <= 256: d <= 128)
  if (tid == 0) last_s = ctas;
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();
  const int unit = __ldcg(&page_rest(part, c)->unit[0]), before = __ldcg(&page_rest(part, c - 1)->unit[1]);
  if (tid + c + 1 < ctas && __ldcg(&page_rest(part, tid + c + 1)->unit[0]) != unit) atomicMin(&last_s, tid + c + 1);  // (fewer CTAs than threads)
  if (unit < 0 || before != unit) return;
  __syncthreads();
  const int last = last_s, share = tid / columns, i = 4 * (tid % columns), g = i / d;
  PageSum sum;
  if (share < shares)
#pragma unroll 1
    for (int z0 = c - 1 + share; z0 < last; z0 += 4 * shares) {
      float m[4], l[4];
      float4 o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int z = min(z0 + k * shares, last - 1);
        const float* p = page_rest_piece(part, ctas, z, z < c ? 1 : 0, per);
        m[k] = __ldcg(p + G * d + g), l[k] = __ldcg(p + G * d + G + g), o[k] = __ldcg(reinterpret_cast<const float4*>(p + i));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (z0 + k * shares < last) sum.add(m[k], l[k], o[k]);
    }
  share_s[tid] = sum;
  __syncthreads();
  if (share == 0) {
    for (int k = 1; k < shares; ++k) sum.add(share_s[columns * k + tid].M, share_s[columns * k + tid].L, share_s[columns * k + tid].O);
    page_emit<ROWS>(a, unit, g, i % d, sum.result());
  }
}

}  // namespace he
