// he_page_append and he_page_read: rows into the pages of a cache of the full history, and back out. Each row is read once and written once, so both are
// bound by HBM (many tokens) or by the latency of a launch and of dependent reads (single tokens).
//
// 8-bit pages hold e4m3 codes and, for K and for V, one scale for each page and KV head, the least power of two with max |x| <= 448 s. With a power
// of two the codes keep the rows' own binary point: code * s is exact in bf16 and fp32, and a scale that grows when a page's later tokens are larger
// moves the codes that are there already by whole binades, which is exact but for those that fall below 2^-6 s, the type's least normal number (rounded once more).
//
// append: a CTA has one page of one sequence (that is, the new rows that lie in it) and walks over KV heads. A thread owns two pieces of a row that hold whole
// rotary pairs, as in rotate_kernel (interleaved pairs are whole in any piece: there the second lies as far on as the first ones of its row's threads reach, so that a warp reads
// and writes whole sectors; 402 MB 69 us, two pieces side by side 100), keeps the sines and cosines of its pairs for all heads, and holds the pieces of K and V in registers from
// the read to the write; between the two lies the maximum over the page, by one barrier a head. Rows into pages of their own type run at HBM's rate (537 MB 84 us, 6.4 TB/s). 8-bit
// pages: some 500 instructions a warp for 32 elements a thread, of rotation, maximum, scaling and conversion, on 67 % of the issue slots: 402 MB 67 us (6.0 TB/s; 63 without a
// rotation; 80 for pages of 128 tokens, one CTA of 1024 threads an SM). 16 ragged prompts of 1024 to 4400 tokens 51 to 53 us, HBM 39: CTAs' starts and the last of 2.3 rounds of them.
// One token of 64 sequences 3.9 us, launch and latency. Where a thread does not hold its place, the sines and, in 8 bits, the rows are fetched and worked out anew for each head and
// pass: 335 MB of fp32 rows into 8-bit pages of 128 tokens 177 us (HBM 51), 402 MB of bf16 at d = 256 327 (62), 402 MB of which 40 of 128 channels turn 235 (62), 537 MB of bf16 at
// d = 256 into pages of their own type 153 (82).
// read: 402 MB of 8-bit pages 64 us (6.3 TB/s).
#pragma once
#include "attend_kernels.cuh"
#include "common.cuh"
#include "rotary_kernels.cuh"

namespace he {

struct AppendArgs {
  he_pages pages;
  const void* x[2];        // k, v
  long long strides[3];    // elements (sequence, head, token)
  const int32_t* new_len;  // [B] or null
  int max_new, n_kv_heads, d;
  int tiles;  // pages that the new rows of a sequence may touch
  int units, heads_per_cta;
  int turns;  // whether keys are rotated; else `rot` says where a thread's pieces lie and nothing more
};

constexpr int kAppendThreads = 1024;  // at most
inline size_t append_smem(int threads) { return (size_t)threads * 2 * 4 * 16; }

// The exponent of the least power of two s >= 2^-100 with top <= 448 s (448 = 1.75 * 2^8), top >= 0 finite and given by its bits.
__host__ __device__ inline int page_scale_exponent(uint32_t top) {
  const int e = (int)(top >> 23) - 127 - ((top & 0x7FFFFFu) <= 0x600000u ? 8 : 7);
  return e > -100 ? e : -100;
}

// A piece over a scale, times inv, as e4m3 codes; what is not finite becomes NaN. Pairs of bf16 values are multiplied as such, which is exact for a power of two but for
// products that are zeros in e4m3 anyway. ANY: inv may be anything, and there may be infinities, which the conversion would saturate.
template <int E, int V, bool ANY>
__device__ __forceinline__ void e4m3_store(uint8_t* dst, RotaryPiece<E, V> p, float inv) {
  uint16_t two[(V + 1) / 2];
  if constexpr (E == 2 && !ANY) {
#pragma unroll
    for (int i = 0; i < p.kWords; ++i) asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(p.w[i]) : "r"(__byte_perm(__float_as_uint(inv), 0, 0x3232)));
    inv = 1.f;
  }
#pragma unroll
  for (int i = 0; i < V; i += 2) {
    float x = p.get(i), y = i + 1 < V ? p.get((i + 1) % V) : 0.f;
    if (ANY) x = fabsf(x) < INFINITY ? x : __int_as_float(0x7FC00000), y = fabsf(y) < INFINITY ? y : __int_as_float(0x7FC00000);
    if (E == 4 || ANY) x *= inv, y *= inv;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two[i / 2]) : "f"(y), "f"(x));
  }
  if constexpr (V == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(two[0] | (uint32_t)two[1] << 16, two[2] | (uint32_t)two[3] << 16);
  else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(dst) = two[0] | (uint32_t)two[1] << 16;
  else if constexpr (V == 2) *reinterpret_cast<uint16_t*>(dst) = two[0];
  else *dst = (uint8_t)two[0];
}

// `bytes` codes (a multiple of 16) times a power of two, by the CTA's threads.
__device__ __forceinline__ void e4m3_rescale(uint8_t* codes, int bytes, float ratio) {
  for (int i = 16 * threadIdx.x; i < bytes; i += 16 * blockDim.x) {
    uint4 raw = *reinterpret_cast<const uint4*>(codes + i);
    float f[16];
    page_unpack(raw, ratio, f);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint16_t lo, hi;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(f[4 * k + 1]), "f"(f[4 * k]));
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(f[4 * k + 3]), "f"(f[4 * k + 2]));
      w[k] = lo | (uint32_t)hi << 16;
    }
    *reinterpret_cast<uint4*>(codes + i) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The largest magnitudes seen so far: a pair of bf16 values (of any sign), or an fp32 one; NaNs are passed over, infinities count.
template <int E, int V>
__device__ __forceinline__ void page_top(uint32_t& top, const RotaryPiece<E, V>& p) {
#pragma unroll
  for (int i = 0; i < RotaryPiece<E, V>::kWords; ++i) {
    if constexpr (E == 2) asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(top) : "r"(p.w[i]));
    else top = __float_as_uint(fmaxf(__uint_as_float(top), fabsf(__uint_as_float(p.w[i]))));
  }
}
// The same of the finite ones alone, as the bits of an fp32 number.
template <int E, int V>
__device__ __forceinline__ void page_top_finite(uint32_t& top, const RotaryPiece<E, V>& p) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t bits = __float_as_uint(p.get(i)) & 0x7FFFFFFFu;
    top = max(top, bits < 0x7F800000u ? bits : 0u);
  }
}

// A row of a page and the two pieces of it that one thread owns.
struct AppendPlace {
  int u, row, c0, c1;
  bool some, second, turns;  // whether there is such a row, a second piece, pairs in them
};

// Interleaved pairs of two pieces, turned: of the first piece by the sines that come first. pair0, pair1: the pieces' first pairs; those from `half` on stay.
template <int E, int V>
__device__ __forceinline__ void page_turn_neighbours(RotaryPiece<E, V>& p0, RotaryPiece<E, V>& p1, const float (&sn)[V], const float (&cs)[V], int pair0, int pair1, int half) {
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    RotaryPiece<E, V>& p = e ? p1 : p0;
    const int left = half - (e ? pair1 : pair0);
    float x[V];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const int k = (e * V + i) / 2;
      const float f = p.get(i), g = p.get(i + 1);
      x[i] = f * cs[k] - g * sn[k], x[i + 1] = g * cs[k] + f * sn[k];
    }
    if (left >= V / 2) {
      p.put(x);
    } else if (left > 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = i / 2 < left ? x[i] : p.get(i);
      p.put(x);
    }
  }
}

// grid.x: pages of sequences, grid.y: shares of the KV heads. With HOLD a thread owns one place of the page, whose pieces of 16 bytes it asks for a head ahead (into
// shared memory that it alone reads) and holds until they are written; without (smaller pieces, pages of more than 1024 places) it walks over as many places as there are,
// twice where the maximum has to be known first.
template <int E, int V, bool INTER, bool Q8, bool HOLD>
__global__ void __launch_bounds__(kAppendThreads) page_append_kernel(const AppendArgs a, const __grid_constant__ he_rotary rot) {
  using Piece = RotaryPiece<E, V>;
  __shared__ uint32_t top_s[3][2][kAppendThreads / 32];
  extern __shared__ __align__(16) uint4 append_s[];  // HOLD: [2][4][threads]
  const he_pages& pg = a.pages;
  const int tid = threadIdx.x, threads = blockDim.x, P = pg.page_size, H = a.n_kv_heads;
  const int s = blockIdx.x / a.tiles;
  griddep_wait();
  griddep_launch_dependents();  // (in this order: a kernel behind this one finds no L1 line of one before it)
  const int held = max(pg.len[s], 0), fresh = a.new_len != nullptr ? min(max(a.new_len[s], 0), a.max_new) : a.max_new;
  const int first = held - fresh;  // the position of row 0; rows ahead of position 0 or behind the table's end are dropped
  const int lo = max(first, 0), hi = (int)min((long long)held, page_capacity(pg));
  const int log2 = __ffs(P) - 1, at = (lo >> log2) + (int)(blockIdx.x - s * a.tiles);
  if (lo >= hi || at > (hi - 1) >> log2) return;
  const int page = page_of(pg, s, at * P);
  if (page < 0) return;
  const int r0 = max(lo - at * P, 0), r1 = min(hi - at * P, P), items = (r1 - r0) * a.units;
  const int half = rot.channels / 2;
  auto place = [&](int item) {
    AppendPlace p;
    const int row = (int)((unsigned)item / (unsigned)a.units);
    p.u = item - row * a.units, p.row = r0 + row, p.some = item < items, p.turns = V * p.u < half;
    p.c0 = INTER ? V * p.u : p.turns ? V * p.u : rot.channels + 2 * V * (p.u - half / V);
    p.c1 = INTER ? p.c0 + V * a.units : p.turns ? p.c0 + half : p.c0 + V;
    p.second = p.some && p.c1 < a.d;
    return p;
  };
  float sn[V], cs[V];
  auto sines = [&](const AppendPlace& p) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int pair = !INTER ? V * p.u + i : i < V / 2 ? p.c0 / 2 + i : p.c1 / 2 + i - V / 2;
      sn[i] = 0.f, cs[i] = 1.f;
      if (a.turns && p.some && pair < half) rotary_sincos(rot, pair, at * P + p.row, sn[i], cs[i]);
    }
  };
  auto turn = [&](const AppendPlace& p, Piece (&x)[2]) {
    if constexpr (INTER) page_turn_neighbours<E, V>(x[0], x[1], sn, cs, p.c0 / 2, p.c1 / 2, half);
    else rotary_turn<E, V, false>(x[0], x[1], sn, cs, p.u, half, p.turns);
  };
  auto read = [&](const AppendPlace& p, int w, int h, Piece (&x)[2]) {
    const char* src = static_cast<const char*>(a.x[w]) + (s * a.strides[0] + h * a.strides[1] + (long long)(at * P + p.row - first) * a.strides[2]) * E;
    if (p.some) x[0].load(src + p.c0 * E);
    if (p.second) x[1].load(src + p.c1 * E);
  };
  auto write = [&](const AppendPlace& p, const Piece (&x)[2], char* to, float inv, auto any) {  // to: the first piece's place in the page
    constexpr int kBytes = Q8 ? 1 : E;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (e ? p.second : p.some) {
        char* at = e ? to + (p.c1 - p.c0) * kBytes : to;
        if constexpr (Q8) e4m3_store<E, V, decltype(any)::value>(reinterpret_cast<uint8_t*>(at), x[e], inv);
        else x[e].store(at);
      }
  };
  auto offset = [&](const AppendPlace& p) { return (p.row * a.d + p.c0) * (Q8 ? 1 : E); };
  const AppendPlace mine = place(tid);
  const int h_begin = blockIdx.y * a.heads_per_cta, h_end = min(h_begin + a.heads_per_cta, H);
  // HOLD: where the next head's pieces are asked from, and the places for them, by turns. (Kept from head to head: worked out anew they were a third of the instructions.)
  const char* next[2];
  const long long from = s * a.strides[0] + h_begin * a.strides[1] + (long long)(at * P + mine.row - first) * a.strides[2] + mine.c0;
  next[0] = static_cast<const char*>(a.x[0]) + from * E, next[1] = static_cast<const char*>(a.x[1]) + from * E;
  const long long head_bytes = a.strides[1] * E;
  const int gap = (mine.c1 - mine.c0) * E;
  uint4* const held_s = append_s + tid;
  char* dst[2];  // the page's rows of this head, with HOLD the thread's first piece of them
  const int page_bytes = P * a.d * (Q8 ? 1 : E);
  {
    const long long begin = ((long long)page * H + h_begin) * page_bytes + (HOLD ? offset(mine) : 0);
    dst[0] = static_cast<char*>(pg.k_pages) + begin, dst[1] = static_cast<char*>(pg.v_pages) + begin;
  }
  auto ask = [&](int h) {
    if (h < h_end) {
      uint4* to = held_s + ((h & 1) ? 4 * threads : 0);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if (mine.some) cp_async16(to + 2 * w * threads, next[w]);
        if (mine.second) cp_async16(to + (2 * w + 1) * threads, next[w] + gap);
        next[w] += head_bytes;
      }
    }
    cp_async_commit();
  };
  if (HOLD) ask(h_begin), sines(mine);
  for (int h = h_begin; h < h_end; ++h, dst[0] += page_bytes, dst[1] += page_bytes) {
    const long long block = (long long)page * H + h;  // of the pages' heads
    float old[2] = {0.f, 0.f};
    if (Q8 && r0 > 0) old[0] = __ldcg(pg.k_scale + block), old[1] = __ldcg(pg.v_scale + block);
    Piece x[2][2];
    uint32_t top[2] = {0u, 0u};
    auto look = [&](const AppendPlace& p, int w, const Piece (&y)[2], bool odd) {
      if (p.some) odd ? page_top_finite(top[w], y[0]) : page_top(top[w], y[0]);
      if (p.second) odd ? page_top_finite(top[w], y[1]) : page_top(top[w], y[1]);
    };
    // the rows of a place as they go into the page
    auto fetch = [&](const AppendPlace& p) {
      read(p, 0, h, x[0]), read(p, 1, h, x[1]);
      if (a.turns && p.some) {
        sines(p);
        turn(p, x[0]);
      }
    };
    if constexpr (HOLD) {
      ask(h + 1);
      cp_async_wait_pending(1);
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int e = 0; e < 2; ++e) x[w][e].load(reinterpret_cast<const char*>(held_s + ((h & 1) ? 4 * threads : 0) + (2 * w + e) * threads));
      if (a.turns && mine.some) turn(mine, x[0]);
      if (Q8) look(mine, 0, x[0], false), look(mine, 1, x[1], false);
      else write(mine, x[0], dst[0], 1.f, std::false_type()), write(mine, x[1], dst[1], 1.f, std::false_type());
    } else {
      for (int item = tid; item < items; item += threads) {
        const AppendPlace p = place(item);
        fetch(p);
        if (Q8) look(p, 0, x[0], false), look(p, 1, x[1], false);
        else write(p, x[0], dst[0] + offset(p), 1.f, std::false_type()), write(p, x[1], dst[1] + offset(p), 1.f, std::false_type());
      }
    }
    if constexpr (!Q8) continue;
    // over the CTA, as the bits of fp32 numbers
    auto gather = [&](int turn) {
      top[0] = __reduce_max_sync(0xFFFFFFFFu, top[0]), top[1] = __reduce_max_sync(0xFFFFFFFFu, top[1]);
      if (threads > 32) {  // (by turns: one barrier a head)
        const int lane = tid & 31;
        if (lane == 0) top_s[turn][0][tid >> 5] = top[0], top_s[turn][1][tid >> 5] = top[1];
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 2; ++w) top[w] = __reduce_max_sync(0xFFFFFFFFu, lane < threads / 32 ? top_s[turn][w][lane] : 0u);
      }
    };
    if (E == 2) top[0] = max(top[0] << 16 & 0x7FFF0000u, top[0] & 0x7FFF0000u), top[1] = max(top[1] << 16 & 0x7FFF0000u, top[1] & 0x7FFF0000u);
    gather(h & 1);
    const bool odd = max(top[0], top[1]) >= 0x7F800000u;  // an infinity (of the whole CTA): the largest of the others is to be found
    if (__builtin_expect(odd, 0)) {
      top[0] = top[1] = 0u;
      if constexpr (HOLD) {
        look(mine, 0, x[0], true), look(mine, 1, x[1], true);
      } else {
        for (int item = tid; item < items; item += threads) {
          const AppendPlace p = place(item);
          fetch(p);
          look(p, 0, x[0], true), look(p, 1, x[1], true);
        }
      }
      gather(2);
      if (threads > 32) __syncthreads();  // (the third place is used by any head)
    }
    float inv[2];
    bool others = odd;  // or an earlier scale that is no power of two
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const int e = page_scale_exponent(top[w]);
      float scale = __int_as_float((127 + e) << 23);
      inv[w] = __int_as_float((127 - e) << 23);
      if (old[w] > scale) scale = old[w], inv[w] = 1.f / scale, others |= (__float_as_uint(inv[w]) & 0x7FFFFFu) != 0u;
      if (r0 > 0 && old[w] != scale) e4m3_rescale(reinterpret_cast<uint8_t*>(dst[w] - (HOLD ? offset(mine) : 0)), r0 * a.d, old[w] / scale);
      if (tid == 0 && (r0 == 0 || old[w] != scale)) (w ? pg.v_scale : pg.k_scale)[block] = scale;
    }
    auto finish = [&](auto any) {
      if constexpr (HOLD) {
        write(mine, x[0], dst[0], inv[0], any), write(mine, x[1], dst[1], inv[1], any);
      } else {
        for (int item = tid; item < items; item += threads) {
          const AppendPlace p = place(item);
          fetch(p);
          write(p, x[0], dst[0] + offset(p), inv[0], any), write(p, x[1], dst[1] + offset(p), inv[1], any);
        }
      }
    };
    if (__builtin_expect(others, 0)) finish(std::true_type());
    else finish(std::false_type());
  }
}

struct ReadArgs {
  he_pages pages;
  void* out[2];         // of k, of v
  long long strides[3];
  const int32_t* first;  // [B] or null
  int max_rows, n_kv_heads, d, sides, side;
};

constexpr int kReadThreads = 256, kReadUnroll = 4, kReadRows = 64;

// 64 positions of a sequence a CTA, one KV head of K or of V, threads (chunk of 16 bytes, row). grid.x: blocks of positions from the first row's on, grid.y: KV heads of K
// and of V, grid.z: sequences.
template <int E, bool Q8>
__global__ void __launch_bounds__(kReadThreads) page_read_kernel(const ReadArgs a) {
  constexpr int N = 16 / E;  // elements
  const he_pages& pg = a.pages;
  const int s = blockIdx.z, h = blockIdx.y % a.n_kv_heads, w = a.sides == 2 ? blockIdx.y / a.n_kv_heads : a.side, c = threadIdx.x * N, P = pg.page_size;
  griddep_wait();
  griddep_launch_dependents();  // (in this order: a kernel behind this one finds no L1 line of one before it)
  const int first = a.first != nullptr ? max(a.first[s], 0) : 0, end = (int)min((long long)page_length(pg, s), (long long)first + a.max_rows);
  const int block = (first / kReadRows + blockIdx.x) * kReadRows;  // (first < end < 2^24 wherever it is used)
  if (first >= end || block >= end) return;
  const char* pages = static_cast<const char*>(w ? pg.v_pages : pg.k_pages);
  const float* scales = w ? pg.v_scale : pg.k_scale;
  char* out = static_cast<char*>(a.out[w]) + (s * a.strides[0] + h * a.strides[1] + c) * E;
  for (int j0 = block + threadIdx.y; j0 < min(block + kReadRows, end); j0 += kReadUnroll * blockDim.y) {
    int page[kReadUnroll];
    uint4 v[kReadUnroll];
    float scale[kReadUnroll];
    auto at = [&](int k) { return j0 + k * (int)blockDim.y; };
    auto some = [&](int k) { return at(k) >= first && at(k) < min(block + kReadRows, end); };
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) page[k] = some(k) ? page_of(pg, s, at(k)) : -1;
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) {
      v[k] = make_uint4(0u, 0u, 0u, 0u), scale[k] = 0.f;
      if (page[k] < 0) continue;
      const long long rows = (long long)page[k] * a.n_kv_heads + h, from = (rows * P + (at(k) & (P - 1))) * a.d + c;
      if constexpr (!Q8) {
        v[k] = ldg_stream16(reinterpret_cast<const uint4*>(pages + from * E));
      } else {
        scale[k] = __ldcg(scales + rows);
        if constexpr (N == 8) {
          const uint2 r = __ldcs(reinterpret_cast<const uint2*>(pages + from));
          v[k].x = r.x, v[k].y = r.y;
        } else {
          v[k].x = __ldcs(reinterpret_cast<const uint32_t*>(pages + from));
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) {
      if (!some(k)) continue;
      uint4 r = v[k];
      if constexpr (Q8) {
        float f[16];
        page_unpack(v[k], scale[k], f);  // (zeros times zero where the page is not there)
        RotaryPiece<E, N> p;
        float g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = f[i];
        p.put(g);
        r = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
      }
      __stcs(reinterpret_cast<uint4*>(out + (long long)(at(k) - first) * a.strides[2] * E), r);
    }
  }
}

}  // namespace he
