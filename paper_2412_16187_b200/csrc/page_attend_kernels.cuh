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

constexpr int kPageWarps = 8, kPageThreads = 32 * kPageWarps, kPageGroup = 32;  // tokens of a group
constexpr int kPageRing = 24 * 1024;                                             // bytes of a warp's ring

struct PageMaps {
  alignas(64) CUtensorMap k, v;
};

template <int D, bool Q8>
struct PageRing {
  static constexpr int kRowBytes = Q8 ? D : 2 * D, kItemBytes = kPageGroup * kRowBytes, kBufs = kPageRing / kItemBytes;
};
inline size_t page_part_floats(int G, int d) { return (size_t)G * (d + 2); }  // of a unit's piece: [G] maxima, [G] sums, [G][d] outputs
inline size_t page_attend_smem(int G, int d) { return 1024 + (size_t)kPageWarps * kPageRing + kPageWarps * page_part_floats(G, d) * sizeof(float); }

// The tokens [lo, hi) that the query of a sequence sees, and their groups [g0, g1).
struct PageSpan {
  int lo, hi, g0, g1;
};
__device__ __forceinline__ PageSpan page_span(const PagedAttendArgs& a, int s) {
  PageSpan p;
  p.hi = page_length(a.pages, s);
  p.lo = a.mod.first_pos != nullptr ? max(a.mod.first_pos[s], 0) : 0;
  if (a.mod.window > 0) p.lo = max(p.lo, p.hi - a.mod.window);
  p.lo = min(p.lo, p.hi);
  p.g0 = p.lo / kPageGroup, p.g1 = p.lo < p.hi ? (p.hi + kPageGroup - 1) / kPageGroup : p.g0;
  return p;
}

// How the line of groups is cut. A thread of the CTA knows the sequences [first, last), whose groups are [base, base + sum) of the line.
struct PageLine {
  long long total, base, sum;
  int parts, first, last;  // parts: CTAs that have some, no fewer than a group per warp each
  __device__ __forceinline__ long long begin(long long part) const { return total * part / parts; }
};
template <typename F>
__device__ __forceinline__ PageLine page_line(const PagedAttendArgs& a, int ctas, long long (&scan_s)[kPageWarps], F empty) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = a.cfg.batch, each = (B + kPageThreads - 1) / kPageThreads;
  PageLine line;
  line.first = min(tid * each, B), line.last = min(line.first + each, B), line.sum = 0, line.base = 0, line.total = 0;
  for (int s = line.first; s < line.last; ++s) {
    const PageSpan p = page_span(a, s);
    line.sum += (long long)(p.g1 - p.g0) * a.cfg.n_kv_heads;
    if (p.g1 == p.g0) empty(s);
  }
  long long incl = line.sum;
#pragma unroll
  for (int off = 1; off < 32; off *= 2) {
    const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, off);
    if (lane >= off) incl += up;
  }
  if (lane == 31) scan_s[warp] = incl;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPageWarps; ++w) {
    if (w < warp) line.base += scan_s[w];
    line.total += scan_s[w];
  }
  line.base += incl - line.sum;
  line.parts = (int)max(1LL, min((long long)ctas, (line.total + kPageWarps - 1) / kPageWarps));
  return line;
}
// The sequence that holds group `at` of the line, and the group's number among those of the sequence (one KV head's after another's): told by the thread that knows it.
template <typename F>
__device__ __forceinline__ void page_find(const PagedAttendArgs& a, const PageLine& line, long long at, F found) {
  at -= line.base;
  if (at < 0 || at >= line.sum) return;
  for (int s = line.first; s < line.last; ++s) {
    const PageSpan p = page_span(a, s);
    const long long n = (long long)(p.g1 - p.g0) * a.cfg.n_kv_heads;
    if (at < n) {
      found(s, at);
      return;
    }
    at -= n;
  }
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

// Folds n pieces into a unit's result or into one piece. get(e, i): number i of piece e, which holds [G] maxima in log2 units, [G] sums, [G][d] outputs.
template <typename F>
__device__ __forceinline__ void page_fold(int n, F get, int G, int d, float* out, float* piece) {
  for (int idx = threadIdx.x; idx < G * d; idx += kPageThreads) {
    const int g = idx / d;
    float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll 4
    for (int e = 0; e < n; ++e) M = fmaxf(M, get(e, g));
#pragma unroll 4
    for (int e = 0; e < n; ++e) {
      const float m = get(e, g), f = m == -INFINITY ? 0.f : exp2f(m - M);
      L += get(e, G + g) * f, O += get(e, 2 * G + idx) * f;
    }
    if (out != nullptr) {
      out[idx] = L != 0.f ? O / L : 0.f;
    } else {
      if (idx % d == 0) piece[g] = M, piece[G + g] = L;
      piece[2 * G + idx] = O;
    }
  }
}

// A place on the line: group g of unit (s, h).
struct PageCursor {
  int s, h, g;
  PageSpan span;
};

// NBOX: pages of a group (2 for pages of 16 tokens). LO: the queries come in fp32 (8-bit pages). FOLD: G <= 4 (bf16 pages).
template <int D, bool Q8, int NBOX, bool LO, bool FOLD>
__global__ void __launch_bounds__(kPageThreads, 1) page_attend_kernel(const __grid_constant__ PagedAttendArgs a, float* part, const __grid_constant__ PageMaps maps) {
  using Ring = PageRing<D, Q8>;
  constexpr int NBUF = Ring::kBufs, ITEM = Ring::kItemBytes, GRP = kPageGroup, NH = Q8 ? 1 : D / 64, SLOTS = NBUF / 2;
  constexpr int NT = D / 8;  // output tiles of 8 channels
  extern __shared__ __align__(16) unsigned char page_smem_raw[];
  __shared__ __align__(8) unsigned long long ring_bar[kPageWarps][NBUF];
  __shared__ float scale_s[kPageWarps][SLOTS][4];  // of the groups under way: K's of each box, V's of each
  __shared__ int ent_unit[2 * kPageWarps], ent_flag[2 * kPageWarps], start_seq[kPageWarps];
  __shared__ long long start_at[kPageWarps], scan_s[kPageWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const he_pages& pg = a.pages;
  const int H = a.cfg.n_kv_heads, G = a.cfg.group_size, d = a.cfg.head_dim, P = pg.page_size;
  unsigned char* smem = page_smem_raw + ((1024u - ((uint32_t)__cvta_generic_to_shared(page_smem_raw) & 1023u)) & 1023u);
  unsigned char* ring = smem + warp * kPageRing;
  const int per = G * (d + 2);
  float* head_piece = reinterpret_cast<float*>(smem + kPageWarps * kPageRing) + warp * per;
  float* tail_piece = reinterpret_cast<float*>(ring);
  auto full = [&](int b) { return (uint32_t)__cvta_generic_to_shared(&ring_bar[warp][b]); };
  if (lane == 0) {
#pragma unroll
    for (int b = 0; b < NBUF; ++b) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(full(b)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    ent_unit[2 * warp] = ent_unit[2 * warp + 1] = -1;
  }
  griddep_wait();
  griddep_launch_dependents();  // (in this order: page_join_kernel reads lengths ahead of its own wait)
  // ---- the work: this CTA's part of the line, and where its warps begin
  const PageLine line = page_line(a, gridDim.x, scan_s, [&](int s) {
    if (s % (int)gridDim.x == (int)blockIdx.x)
      for (int i = 0; i < H * G * d; i += 4) *reinterpret_cast<float4*>(a.out + (long long)s * H * G * d + i) = make_float4(0.f, 0.f, 0.f, 0.f);
  });
  if ((int)blockIdx.x >= line.parts) return;
  const long long begin = line.begin(blockIdx.x), end = line.begin(blockIdx.x + 1);
  auto warp_begin = [&](int w) { return begin + (end - begin) * w / kPageWarps; };
#pragma unroll 1
  for (int w = 0; w < kPageWarps; ++w)
    if (warp_begin(w) < end) page_find(a, line, warp_begin(w), [&](int s, long long at) { start_seq[w] = s, start_at[w] = at; });
  __syncthreads();
  const int groups = (int)(warp_begin(warp + 1) - warp_begin(warp)), items = 2 * groups;
  PageCursor cur{}, ask{};  // the group that is worked on, the one that is asked for next
  if (groups > 0) {
    cur.s = start_seq[warp], cur.span = page_span(a, cur.s);
    const int n = cur.span.g1 - cur.span.g0;
    cur.h = (int)(start_at[warp] / n), cur.g = cur.span.g0 + (int)(start_at[warp] % n);
    ask = cur;
  }
  auto advance = [&](PageCursor& c) {
    if (++c.g < c.span.g1) return;
    if (++c.h == H) {
      c.h = 0;
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
  auto issue = [&](int t, int b) {
    if (t >= items) return;
    int row[NBOX];
#pragma unroll
    for (int i = 0; i < NBOX; ++i) {
      const int p = __shfl_sync(0xFFFFFFFFu, page, i);
      row[i] = p < 0 ? none : (p * H + ask.h) * P + (ask.g * GRP + 16 * i) % P;
    }
    if (lane == 0) {
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(ring + b * ITEM);
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full(b)), "r"((uint32_t)ITEM) : "memory");
#pragma unroll
      for (int i = 0; i < NBOX; ++i)
#pragma unroll
        for (int h = 0; h < NH; ++h)
          asm volatile(
              "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                  dst + h * GRP * 128 + i * (GRP / NBOX) * (Ring::kRowBytes / NH)),
              "l"(reinterpret_cast<uint64_t>((t & 1) ? &maps.v : &maps.k)), "r"(h * 64), "r"(row[i]), "r"(full(b))
              : "memory");
    }
    if ((t & 1) == 0) {
      if (Q8) scale = lane < 4 && page >= 0 ? __ldcg((lane < 2 ? pg.k_scale : pg.v_scale) + (long long)page * H + ask.h) : 0.f;
    } else {
      if (Q8 && lane < 4) scale_s[warp][(t >> 1) % SLOTS][lane] = scale;
      if (t + 1 < items) {
        advance(ask);
        look_up();
      }
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
  constexpr int OW = Q8 ? 2 : 4;
  float m = -INFINITY, l = 0.f, o[NT][OW];
  auto clear = [&]() {
    m = -INFINITY, l = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < OW; ++e) o[t][e] = 0.f;
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
#pragma unroll 1
  for (int t = 0; t < items && ok; t += 2) {
    if (fresh) load_q(), begins = cur.g == cur.span.g0, fresh = false;
    const int j0 = cur.g * GRP, lo = cur.span.lo, hi = cur.span.hi;
    float sa[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sa[i][e] = 0.f;
    float sb[4][4];
    if constexpr (!Q8) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sb[i][e] = 0.f;
    }
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    {
      const unsigned char* tile = step(t);
      if constexpr (Q8) {
        __syncwarp();
#pragma unroll
        for (int b = 0; b < NBOX; ++b) ks[b] = scale_s[warp][(t >> 1) % SLOTS][b], vs[b] = scale_s[warp][(t >> 1) % SLOTS][2 + b];
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 kv = *reinterpret_cast<const uint4*>(code_at(tile, 8 * i + gid, D == 128 ? 2 * tig + c : tig));
            const uint32_t w[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
            for (int u = 0; u < 4; ++u)
              mma_f16_m16n8k16(sa[i], qf[8 * c + 2 * u], LO ? ql[LO ? 8 * c + 2 * u : 0] : 0u, qf[8 * c + 2 * u + 1], LO ? ql[LO ? 8 * c + 2 * u + 1 : 0] : 0u,
                               e4m3_halves(w[u] & 0xFFFFu), e4m3_halves(w[u] >> 16));
          }
      } else {
        const uint4* kr = reinterpret_cast<const uint4*>(tile) + gid * 8;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 kv = kr[(c >> 1) * GRP * 8 + i * 64 + ((2 * tig + (c & 1)) ^ gid)];
            mma_bf16_m16n8k16(sa[i], qf[4 * c], 0u, qf[4 * c + 1], 0u, kv.x, kv.y);
            mma_bf16_m16n8k16(sb[i], qf[4 * c + 2], 0u, qf[4 * c + 3], 0u, kv.z, kv.w);
          }
      }
    }
    // This lane: head gid, tokens j0 + 8 i + 2 tig, + 1.
    const uint32_t seen = (lo > j0 ? 0xFFFFFFFFu << (lo - j0) : 0xFFFFFFFFu) & (hi < j0 + 32 ? (1u << (hi - j0)) - 1u : 0xFFFFFFFFu);
    float x[8], gm = -INFINITY;
    const float away = (float)(hi - 1 - j0 - 2 * tig);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float kscale = ks[NBOX == 2 ? i >> 1 : 0];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float dot = Q8 ? (LO ? sa[i][e] + sa[i][2 + e] : sa[i][e]) : sa[i][e] + sb[i][e];
        float y = a.mod.cap_log2 > 0.f ? a.mod.cap_log2 * tanhf(dot * (inv_cap * kscale)) : dot * (factor * kscale);
        y = fmaf(-slope, fabsf(away - (float)(8 * i + e)), y);
        x[2 * i + e] = (seen >> (8 * i + 2 * tig + e)) & 1u ? y : -INFINITY;
        gm = fmaxf(gm, x[2 * i + e]);
      }
    }
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 1));
    gm = fmaxf(gm, __shfl_xor_sync(0xFFFFFFFFu, gm, 2));
    constexpr float kUp = Q8 ? 14.f : 0.f;  // weights times 2^14: sums and outputs alike
    const float mx = fmaxf(m, gm), mn = mx == -INFINITY ? 0.f : mx;
    const float corr = page_ex2(m - mn);
    float p[8], ps = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = page_ex2(x[k] - mn + kUp);
#pragma unroll
    for (int k = 0; k < 8; k += 2) ps += p[k] + p[k + 1];
    l = l * corr + ps;
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
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        o[u][0] *= corr, o[u][1] *= corr;
        if constexpr (!Q8) o[u][OW - 2] *= corr, o[u][OW - 1] *= corr;
      }
    }
    const unsigned char* tile = step(t + 1);
    if constexpr (Q8) {
#pragma unroll
      for (int b = 0; b < NBOX; ++b)
        if (NBOX == 2 && ((seen >> (16 * b)) & 0xFFFFu) == 0u) vs[b] = 0.f;  // (a page that is not seen has any scale)
      constexpr int WORDS = D / 32;  // of a lane's D / 8 codes of a row
      uint32_t v[2][4][WORDS];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int row = 16 * hf + 2 * tig + (s & 1) + 8 * (s >> 1);
          if constexpr (D == 128) {
            const uint4 r = *reinterpret_cast<const uint4*>(code_at(tile, row, gid));
            v[hf][s][0] = r.x, v[hf][s][1] = r.y, v[hf][s][WORDS - 2] = r.z, v[hf][s][WORDS - 1] = r.w;
          } else {
            const uint2 r = *reinterpret_cast<const uint2*>(code_at(tile, row, gid >> 1) + 8 * (gid & 1));
            v[hf][s][0] = r.x, v[hf][s][1] = r.y;
          }
          if (seen != 0xFFFFFFFFu) {  // hidden rows (weighted by zero) hold anything: zeros
#pragma unroll
            for (int q = 0; q < WORDS; ++q) v[hf][s][q] &= 0u - ((seen >> row) & 1u);
          }
        }
      float c[NBOX][4][4];
#pragma unroll
      for (int q = 0; q < WORDS; ++q) {  // four channels of each lane column at a time: tiles 4 q .. 4 q + 3
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          // codes of two tokens by channel
          const uint32_t a01 = __byte_perm(v[hf][0][q], v[hf][1][q], 0x5140u), a23 = __byte_perm(v[hf][0][q], v[hf][1][q], 0x7362u);
          const uint32_t b01 = __byte_perm(v[hf][2][q], v[hf][3][q], 0x5140u), b23 = __byte_perm(v[hf][2][q], v[hf][3][q], 0x7362u);
          const int set = NBOX == 2 ? hf : 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (NBOX == 2 || hf == 0) c[set][e][0] = c[set][e][1] = c[set][e][2] = c[set][e][3] = 0.f;
            const uint32_t first = e < 2 ? a01 : a23, second = e < 2 ? b01 : b23;
            mma_f16_m16n8k16(c[set][e], w[2 * hf][0], w[2 * hf][1], w[2 * hf + 1][0], w[2 * hf + 1][1], e4m3_halves((e & 1) ? first >> 16 : first & 0xFFFFu),
                             e4m3_halves((e & 1) ? second >> 16 : second & 0xFFFFu));
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            o[4 * q + e][k] = fmaf(c[0][e][k] + c[0][e][2 + k], vs[0], o[4 * q + e][k]);
            if constexpr (NBOX == 2) o[4 * q + e][k] = fmaf(c[1][e][k] + c[1][e][2 + k], vs[1], o[4 * q + e][k]);
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
            const int row = 16 * hf + 2 * tig + (s & 1) + 8 * (s >> 1);
            vb[hf][s] = vr[h * GRP * 8 + row * 8 + (gid ^ (row & 7))];
          }
        if (seen != 0xFFFFFFFFu) {
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
          for (int k = 0; k < 4; ++k) o[8 * h + e][k % OW] += c[k];
        }
      }
    }
    const bool ends = cur.g + 1 == cur.span.g1;
    if (ends || t + 2 == items) {  // the unit's result, or this warp's piece of it
      l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
      l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
      if constexpr (!Q8) {
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (FOLD) o[u][k] += __shfl_down_sync(0xFFFFFFFFu, o[u][k], 16);  // the third terms' share
            o[u][k] += o[u][OW - 2 + k];
          }
      }
      const bool whole = begins && ends;
      float* dst = whole ? a.out + ((long long)cur.s * H + cur.h) * G * d : (ends ? head_piece : tail_piece) + 2 * G;
      const float inv = whole ? (l != 0.f ? 1.f / l : 0.f) : 1.f;
      __syncwarp();  // (the ring has been read: its first bytes take the last piece)
      if (gid < G) {
        if (!whole && tig == 0) dst[gid - 2 * G] = m, dst[gid - G] = l;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int n = 2 * tig + k;  // lane column
          if constexpr (Q8) {  // channels n * D / 8 + u
#pragma unroll
            for (int u = 0; u < NT; u += 4)
              if (n * NT + u < d) {
                const float f[4] = {o[u][k] * inv, o[u + 1][k] * inv, o[u + 2][k] * inv, o[u + 3][k] * inv};
                float* to = dst + gid * d + n * NT + u;
                if (whole) *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
                else to[0] = f[0], to[1] = f[1], to[2] = f[2], to[3] = f[3];
              }
          } else {  // channels (n + 8 h) * 8 + e of tile 8 h + e
#pragma unroll
            for (int u = 0; u < NT; u += 4) {
              const int ch = (n + 8 * (u >> 3)) * 8 + (u & 7);
              if (ch < d) {
                const float f[4] = {o[u][k] * inv, o[u + 1][k] * inv, o[u + 2][k] * inv, o[u + 3][k] * inv};
                float* to = dst + gid * d + ch;
                if (whole) *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
                else to[0] = f[0], to[1] = f[1], to[2] = f[2], to[3] = f[3];
              }
            }
          }
        }
      }
      if (!whole && lane == 0) {
        const int e = 2 * warp + (ends ? 0 : 1);
        ent_unit[e] = cur.s * H + cur.h, ent_flag[e] = (begins ? 1 : 0) | (ends ? 2 : 0);
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
  // ---- units that several warps share
  const float* heads = reinterpret_cast<const float*>(smem + kPageWarps * kPageRing);
#pragma unroll 1
  for (int e = 0; e < 2 * kPageWarps;) {
    if (ent_unit[e] < 0) {
      ++e;
      continue;
    }
    int n = 0, z = e;
    uint32_t bits = 0u;
    for (; z < 2 * kPageWarps && (ent_unit[z] < 0 || ent_unit[z] == ent_unit[e]); ++z)
      if (ent_unit[z] >= 0) bits |= 1u << z, ++n;
    const int last = 31 - __clz(bits), unit = ent_unit[e];
    const bool from_start = ent_flag[e] & 1, to_end = ent_flag[last] & 2;
    auto get = [&](int i, int number) {
      uint32_t rest = bits;
      for (int k = 0; k < i; ++k) rest &= rest - 1u;
      const int at = __ffs(rest) - 1;
      return ((at & 1) ? reinterpret_cast<const float*>(smem + (at >> 1) * kPageRing) : heads + (at >> 1) * per)[number];
    };
    if (from_start && to_end) page_fold(n, get, G, d, a.out + (long long)unit * G * d, nullptr);
    else page_fold(n, get, G, d, nullptr, part + (2 * (long long)blockIdx.x + (from_start ? 1 : 0)) * per);
    e = z;
  }
}

// Units that several CTAs share: the CTA whose part begins in the middle of one, and is the first such, puts its pieces together.
static __global__ void __launch_bounds__(kPageThreads) page_join_kernel(const __grid_constant__ PagedAttendArgs a, const float* part, int ctas) {
  __shared__ long long scan_s[kPageWarps], at_s;
  __shared__ int seq_s;
  const int c = blockIdx.x + 1, H = a.cfg.n_kv_heads, G = a.cfg.group_size, d = a.cfg.head_dim, per = G * (d + 2);
  const PageLine line = page_line(a, ctas, scan_s, [](int) {});
  if (c >= line.parts) return;
  const long long at = line.begin(c);
  page_find(a, line, at, [&](int s, long long in) { seq_s = s, at_s = in; });
  __syncthreads();
  const PageSpan p = page_span(a, seq_s);
  const int n = p.g1 - p.g0, h = (int)(at_s / n);
  const long long unit0 = at - at_s % n, unit1 = unit0 + n;  // the unit's groups on the line
  if (unit0 == at || line.begin(c - 1) > unit0) return;
  int end = c + 1;
  while (end < line.parts && line.begin(end) < unit1) ++end;
  griddep_wait();
  page_fold(end - c + 1, [&](int e, int i) { return __ldcg(part + (2 * (long long)(c - 1 + e) + (e == 0 ? 1 : 0)) * per + i); }, G, d,
            a.out + ((long long)seq_s * H + h) * G * d, nullptr);
}

}  // namespace he
