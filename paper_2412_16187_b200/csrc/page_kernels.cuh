// he_page_append and he_page_read: rows into the pages of a cache of the full history, and back out. Each row is read once and written once, so both are
// bound by HBM (many tokens) or by the latency of a launch and of dependent reads (single tokens).
//
// 8-bit pages hold e4m3 codes and, for K and for V, one scale for each page and KV head, the least power of two with max |x| <= 448 s. With a power
// of two the codes keep the rows' own binary point: code * s is exact in bf16 and fp32, and a scale that grows when a page's later tokens are larger
// moves the codes that are there already by whole binades, which is exact but for those that fall below 2^-6 s, the type's least normal number (rounded once more).
//
// append: a CTA has one page of one sequence (that is, the new rows that lie in it) and walks over KV heads. A thread owns two pieces of a row that hold whole
// rotary pairs, as in rotate_kernel, keeps the sines and cosines of its pairs for all heads, and holds the pieces of K and V in registers from
// the read to the write; between the two lies the maximum over the page, by one barrier.
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
};

constexpr int kAppendThreads = 512;  // at most
template <int E>
constexpr int kAppendPairs = E == 2 ? 16 : 8;  // of a thread that holds them: what 128 registers take

// The exponent of the least power of two s >= 2^-100 with top <= 448 s (448 = 1.75 * 2^8), top >= 0 finite and given by its bits.
__host__ __device__ inline int page_scale_exponent(uint32_t top) {
  const int e = (int)(top >> 23) - 127 - ((top & 0x7FFFFFu) <= 0x600000u ? 8 : 7);
  return e > -100 ? e : -100;
}

// V values over a scale as e4m3 codes; what is not finite becomes NaN.
template <int V>
__device__ __forceinline__ void e4m3_store(uint8_t* dst, const float (&f)[V], float inv) {
  uint16_t two[(V + 1) / 2];
#pragma unroll
  for (int i = 0; i < V; i += 2) {
    const float x = f[i], y = i + 1 < V ? f[(i + 1) % V] : 0.f;
    const float cx = fabsf(x) < INFINITY ? x * inv : __int_as_float(0x7FC00000), cy = fabsf(y) < INFINITY ? y * inv : __int_as_float(0x7FC00000);
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two[i / 2]) : "f"(cy), "f"(cx));
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

// The largest of the bits of finite magnitudes, of V values.
template <int E, int V>
__device__ __forceinline__ uint32_t page_top(uint32_t top, const RotaryPiece<E, V>& p) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t bits = __float_as_uint(p.get(i)) & 0x7FFFFFFFu;
    top = max(top, bits < 0x7F800000u ? bits : 0u);
  }
  return top;
}

// A row of a page and the two pieces of it that one thread owns.
struct AppendPlace {
  int u, row, c0, c1;
  bool some, second, turns;  // whether there is such a row, a second piece, pairs in them
};

// grid.x: pages of sequences, grid.y: shares of the KV heads. With HOLD a thread owns pieces of kAppendPairs pairs at most and holds what it has read; without (pieces of fewer
// than 16 bytes, pages too large for 512 threads) it walks over as many as there are, twice where the maximum has to be known first.
template <int E, int V, bool INTER, bool Q8, bool HOLD>
__global__ void __launch_bounds__(kAppendThreads) page_append_kernel(const AppendArgs a, const __grid_constant__ he_rotary rot) {
  using Piece = RotaryPiece<E, V>;
  constexpr int ITEMS = HOLD ? kAppendPairs<E> / V : 1;
  __shared__ uint32_t top_s[2][2][kAppendThreads / 32];
  const he_pages& pg = a.pages;
  const int tid = threadIdx.x, threads = blockDim.x, P = pg.page_size, H = a.n_kv_heads;
  const int s = blockIdx.x / a.tiles;
  griddep_wait();
  griddep_launch_dependents();  // (in this order: a kernel behind this one finds no L1 line of one before it)
  const int held = max(pg.len[s], 0), fresh = a.new_len != nullptr ? min(max(a.new_len[s], 0), a.max_new) : a.max_new;
  const int first = held - fresh;  // the position of row 0; rows ahead of position 0 or behind the table's end are dropped
  const int lo = max(first, 0), hi = (int)min((long long)held, page_capacity(pg));
  const int at = lo / P + (int)(blockIdx.x % a.tiles);
  if (lo >= hi || at > (hi - 1) / P) return;
  const int page = page_of(pg, s, at * P);
  if (page < 0) return;
  const int r0 = max(lo - at * P, 0), r1 = min(hi - at * P, P), items = (r1 - r0) * a.units;
  const int half = rot.channels / 2;
  auto place = [&](int item) {
    AppendPlace p;
    p.u = item % a.units, p.row = r0 + item / a.units, p.some = item < items, p.turns = V * p.u < half;
    p.c0 = INTER ? 2 * V * p.u : p.turns ? V * p.u : rot.channels + 2 * V * (p.u - half / V);
    p.c1 = !INTER && p.turns ? p.c0 + half : p.c0 + V;
    p.second = p.some && p.c1 < a.d;
    return p;
  };
  auto sines = [&](const AppendPlace& p, float (&sn)[V], float (&cs)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sn[i] = 0.f, cs[i] = 1.f;
      if (p.some && V * p.u + i < half) rotary_sincos(rot, V * p.u + i, at * P + p.row, sn[i], cs[i]);
    }
  };
  auto read = [&](const AppendPlace& p, int w, int h, Piece (&x)[2]) {
    const char* src = static_cast<const char*>(a.x[w]) + (s * a.strides[0] + h * a.strides[1] + (long long)(at * P + p.row - first) * a.strides[2]) * E;
    if (p.some) x[0].load(src + p.c0 * E);
    if (p.second) x[1].load(src + p.c1 * E);
  };
  auto write = [&](const AppendPlace& p, const Piece (&x)[2], char* dst, float inv) {  // dst: the page's rows of this head
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (e ? p.second : p.some) {
        const long long to = (long long)p.row * a.d + (e ? p.c1 : p.c0);
        if constexpr (Q8) {
          float f[V];
#pragma unroll
          for (int i = 0; i < V; ++i) f[i] = x[e].get(i);
          e4m3_store<V>(reinterpret_cast<uint8_t*>(dst) + to, f, inv);
        } else {
          x[e].store(dst + to * E);
        }
      }
  };
  AppendPlace mine[ITEMS];
  float sn[ITEMS][V], cs[ITEMS][V];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    mine[k] = place(tid + k * threads);
    if (HOLD) sines(mine[k], sn[k], cs[k]);
  }
  const int h_begin = blockIdx.y * a.heads_per_cta, h_end = min(h_begin + a.heads_per_cta, H);
  for (int h = h_begin; h < h_end; ++h) {
    const long long block = (long long)page * H + h;  // of the pages' heads
    char* dst[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) dst[w] = static_cast<char*>(w ? pg.v_pages : pg.k_pages) + block * P * a.d * (Q8 ? 1 : E);
    float old[2] = {0.f, 0.f};
    if (Q8 && r0 > 0) old[0] = __ldcg(pg.k_scale + block), old[1] = __ldcg(pg.v_scale + block);
    Piece x[2][ITEMS][2];
    uint32_t top[2] = {0u, 0u};
    auto look = [&](const AppendPlace& p, int w, const Piece (&y)[2]) {
      if (p.some) top[w] = page_top(top[w], y[0]);
      if (p.second) top[w] = page_top(top[w], y[1]);
    };
    // the rows of an item as they go into the page
    auto fetch = [&](const AppendPlace& p, Piece (&k)[2], Piece (&v)[2]) {
      read(p, 0, h, k), read(p, 1, h, v);
      if (p.some) {
        sines(p, sn[0], cs[0]);
        rotary_turn<E, V, INTER>(k[0], k[1], sn[0], cs[0], p.u, half, p.turns);
      }
    };
    if constexpr (HOLD) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) read(mine[k], 0, h, x[0][k]), read(mine[k], 1, h, x[1][k]);
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
        if (mine[k].some) rotary_turn<E, V, INTER>(x[0][k][0], x[0][k][1], sn[k], cs[k], mine[k].u, half, mine[k].turns);
      if (!Q8) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) write(mine[k], x[0][k], dst[0], 1.f), write(mine[k], x[1][k], dst[1], 1.f);
      } else {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) look(mine[k], 0, x[0][k]), look(mine[k], 1, x[1][k]);
      }
    } else {
      for (int item = tid; item < items; item += threads) {
        const AppendPlace p = place(item);
        fetch(p, x[0][0], x[1][0]);
        if (Q8) look(p, 0, x[0][0]), look(p, 1, x[1][0]);
        else write(p, x[0][0], dst[0], 1.f), write(p, x[1][0], dst[1], 1.f);
      }
    }
    if constexpr (!Q8) continue;
    top[0] = __reduce_max_sync(0xFFFFFFFFu, top[0]), top[1] = __reduce_max_sync(0xFFFFFFFFu, top[1]);
    if (threads > 32) {  // (by turns: one barrier a head)
      const int lane = tid & 31;
      if (lane == 0) top_s[h & 1][0][tid >> 5] = top[0], top_s[h & 1][1][tid >> 5] = top[1];
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 2; ++w) top[w] = __reduce_max_sync(0xFFFFFFFFu, lane < threads / 32 ? top_s[h & 1][w][lane] : 0u);
    }
    float inv[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float scale = fmaxf(__int_as_float((page_scale_exponent(top[w]) + 127) << 23), old[w]);
      inv[w] = 1.f / scale;
      if (r0 > 0 && old[w] != scale) e4m3_rescale(reinterpret_cast<uint8_t*>(dst[w]), r0 * a.d, old[w] / scale);
      if (tid == 0 && (r0 == 0 || old[w] != scale)) (w ? pg.v_scale : pg.k_scale)[block] = scale;
    }
    if constexpr (HOLD) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) write(mine[k], x[0][k], dst[0], inv[0]), write(mine[k], x[1][k], dst[1], inv[1]);
    } else {
      for (int item = tid; item < items; item += threads) {
        const AppendPlace p = place(item);
        fetch(p, x[0][0], x[1][0]);
        write(p, x[0][0], dst[0], inv[0]), write(p, x[1][0], dst[1], inv[1]);
      }
    }
  }
}

struct ReadArgs {
  he_pages pages;
  void* out[2];         // of k, of v
  long long strides[3];
  const int32_t* first;  // [B] or null
  int max_rows, n_kv_heads, d, sides, side;
};

constexpr int kReadThreads = 256, kReadUnroll = 4;

// 16 bytes of a row at a time. grid.x: rows, grid.y: KV heads of K and of V, grid.z: sequences.
template <int E, bool Q8>
__global__ void __launch_bounds__(kReadThreads) page_read_kernel(const ReadArgs a) {
  constexpr int N = 16 / E;  // elements
  const he_pages& pg = a.pages;
  const int s = blockIdx.z, h = blockIdx.y % a.n_kv_heads, w = a.sides == 2 ? blockIdx.y / a.n_kv_heads : a.side;
  griddep_wait();
  griddep_launch_dependents();  // (in this order: a kernel behind this one finds no L1 line of one before it)
  const int first = a.first != nullptr ? max(a.first[s], 0) : 0, rows = min(page_length(pg, s) - first, a.max_rows), cpr = a.d / N;
  const char* pages = static_cast<const char*>(w ? pg.v_pages : pg.k_pages);
  const float* scales = w ? pg.v_scale : pg.k_scale;
  char* out = static_cast<char*>(a.out[w]) + (s * a.strides[0] + h * a.strides[1]) * E;
  const long long item0 = (long long)blockIdx.x * kReadThreads * kReadUnroll + threadIdx.x;
  if (item0 - threadIdx.x >= (long long)rows * cpr) return;
  int row[kReadUnroll], c[kReadUnroll], page[kReadUnroll];
#pragma unroll
  for (int k = 0; k < kReadUnroll; ++k) {
    const long long item = item0 + k * kReadThreads;
    row[k] = (int)(item / cpr), c[k] = (int)(item % cpr);
    page[k] = row[k] < rows ? page_of(pg, s, first + row[k]) : -1;
  }
  uint4 v[kReadUnroll];
  float scale[kReadUnroll];
#pragma unroll
  for (int k = 0; k < kReadUnroll; ++k) {
    v[k] = make_uint4(0u, 0u, 0u, 0u), scale[k] = 0.f;
    if (page[k] < 0) continue;
    const long long block = (long long)page[k] * a.n_kv_heads + h, at = (block * pg.page_size + (first + row[k]) % pg.page_size) * a.d + c[k] * N;
    if constexpr (!Q8) {
      v[k] = ldg_stream16(reinterpret_cast<const uint4*>(pages + at * E));
    } else {
      scale[k] = __ldcg(scales + block);
      if constexpr (N == 8) {
        const uint2 r = __ldcs(reinterpret_cast<const uint2*>(pages + at));
        v[k].x = r.x, v[k].y = r.y;
      } else {
        v[k].x = __ldcs(reinterpret_cast<const uint32_t*>(pages + at));
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kReadUnroll; ++k) {
    if (row[k] >= rows) continue;
    uint4 r = v[k];
    if constexpr (Q8) {
      float f[16];
      page_unpack(v[k], scale[k], f);
      RotaryPiece<E, N> p;
      float g[N];
#pragma unroll
      for (int i = 0; i < N; ++i) g[i] = page[k] < 0 ? 0.f : f[i];
      p.put(g);
      r = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
    }
    *reinterpret_cast<uint4*>(out + ((long long)row[k] * a.strides[2] + c[k] * N) * E) = r;
  }
}

}  // namespace he
