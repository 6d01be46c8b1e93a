// he_rotate_prompt and he_rotate_step: rotary positions of query and key rows. A pair (a, c) at position p with frequency f becomes
// amplitude * (a cos pf - c sin pf, c cos pf + a sin pf). Each row is read once and written once, so the calls are bound by HBM
// (prompts) and by the latency of a launch and two dependent reads (single tokens).
//
// Angles. A frequency is held as turns per position, modulo one turn, in units of 2^-64 (he_rotary.turns): the product with an
// int32 position in 64-bit integers drops whole turns by itself and is exact, where fp32 would have lost the angle of position
// 10^6 in its second decimal. The upper 32 bits as a signed number are the angle in [-1/2, 1/2) turns, and sincospif takes it from there.
//
// Work. A thread owns two pieces of a row that hold whole pairs: the channels [Vu, Vu + V) and their partners r/2 further in the half
// layout, 2V neighbours in the interleaved one; nobody else touches them, so a call may work in place. A piece is 16 bytes wide where
// r/2 allows it (always in the interleaved layout), else the largest power of two that divides r/2. The thread works out the sines and cosines of its V pairs
// once for a token and walks over heads with them. Channels from r on are copied by threads of their own in the half layout.
//
// Measured: 40 heads of 32768 tokens at d = 128 (671 MB) 108 us, 6.2 TB/s; a step of 256 sequences of 40 heads 8 us, bound by launch and latency.
#pragma once
#include "common.cuh"

namespace he {

struct RotateArgs {
  const void* x[2];  // q, k
  void* y[2];
  long long in[2][3], out[2][3];  // element strides (sequence, head, token)
  int heads[2];                   // of q and of k; 0: not given
  int n_kv_heads, group;
  int d, dtype;
  int batch, tokens;         // tokens per sequence: max_prompt_len, or 1
  const int32_t* positions;  // [B, tokens] or null
  const int32_t* lens;       // [B] or null
  const int32_t* next_pos;   // [B, Hkv] (single tokens) or null
  int units;                 // threads per row
  int heads_per_thread;
};

constexpr int kRotateThreads = 256;

// V elements of E bytes as they lie in memory, and as fp32 (packing rounds once).
template <int E, int V>
struct RotaryPiece {
  static constexpr int kWords = (V * E + 3) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const char* p) {
    if constexpr (V * E == 16) {
      const uint4 r = *reinterpret_cast<const uint4*>(p);
      w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
    } else if constexpr (V * E == 8) {
      const uint2 r = *reinterpret_cast<const uint2*>(p);
      w[0] = r.x, w[1] = r.y;
    } else if constexpr (V * E == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    if constexpr (V * E == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (V * E == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (V * E == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (E == 4) return __uint_as_float(w[i]);
    else return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void put(const float (&f)[V]) {
    if constexpr (E == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(w[i]) : "f"(2 * i + 1 < V ? f[(2 * i + 1) % V] : 0.f), "f"(f[2 * i]));
    }
  }
};

__device__ __forceinline__ void rotary_sincos(const he_rotary& r, int pair, int pos, float& s, float& c) {
  const unsigned long long turn = (unsigned long long)(long long)pos * r.turns[pair];
  sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s, &c);  // half turns
  s *= r.amplitude, c *= r.amplitude;
}

// Elements of a piece: 16 bytes' worth, in the half layout halved until they divide r/2.
inline int rotary_piece(const he_rotary& r, int esize) {
  int v = 16 / esize;
  if (!r.interleaved)
    while ((r.channels / 2) % v != 0) v /= 2;
  return v;
}
// Threads per row.
inline int rotary_units(const he_rotary& r, int d, int v) {
  if (r.interleaved) return (d + 2 * v - 1) / (2 * v);
  return r.channels / 2 / v + (d - r.channels + 2 * v - 1) / (2 * v);
}

// The pairs of a thread's two pieces, turned. u: which pieces of the row; half: pairs of a row; turns: whether they hold any (half layout).
template <int E, int V, bool INTER>
__device__ __forceinline__ void rotary_turn(RotaryPiece<E, V>& p0, RotaryPiece<E, V>& p1, const float (&sn)[V], const float (&cs)[V], int u, int half, bool turns) {
  if (!turns) return;
  float x[V], y[V];
  if (INTER) {  // pairs are neighbours: the first piece's, then the second's; those beyond r stay
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const int j = i / 2, k = (V + i) / 2;
      const float a0 = p0.get(i), b0 = p0.get(i + 1), a1 = p1.get(i), b1 = p1.get(i + 1);
      const bool in0 = V * u + j < half, in1 = V * u + k < half;
      x[i] = in0 ? a0 * cs[j] - b0 * sn[j] : a0, x[i + 1] = in0 ? b0 * cs[j] + a0 * sn[j] : b0;
      y[i] = in1 ? a1 * cs[k] - b1 * sn[k] : a1, y[i + 1] = in1 ? b1 * cs[k] + a1 * sn[k] : b1;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float a0 = p0.get(i), b0 = p1.get(i);
      x[i] = a0 * cs[i] - b0 * sn[i], y[i] = b0 * cs[i] + a0 * sn[i];
    }
  }
  p0.put(x), p1.put(y);
}

// grid.x: threads of (sequence, token, unit), grid.y: shares of the heads (q's first, then k's).
template <int E, int V, bool INTER>
__global__ void __launch_bounds__(kRotateThreads) rotate_kernel(const RotateArgs a, const __grid_constant__ he_rotary rot) {
  using Piece = RotaryPiece<E, V>;
  griddep_launch_dependents();
  griddep_wait();
  const long long item = (long long)blockIdx.x * kRotateThreads + threadIdx.x;
  const int u = (int)(item % a.units);
  const long long row = item / a.units;
  if (row >= (long long)a.batch * a.tokens) return;
  const int s = (int)(row / a.tokens), n = (int)(row % a.tokens);
  if (a.lens != nullptr && n >= a.lens[s]) return;
  const int all = a.heads[0] + a.heads[1];
  const int h_begin = blockIdx.y * a.heads_per_thread, h_end = min(h_begin + a.heads_per_thread, all);
  const int half = rot.channels / 2;
  const bool turns = V * u < half;  // (interleaved: the pieces hold the pairs [Vu, Vu + V), some of them perhaps beyond r)
  const int c0 = INTER ? 2 * V * u : turns ? V * u : rot.channels + 2 * V * (u - half / V);
  const int c1 = !INTER && turns ? c0 + half : c0 + V;
  const bool second = c1 < a.d;
  float sn[V], cs[V];
  // (single tokens: a thread has one head, whose unit says the position)
  const int unit = h_begin >= a.heads[0] ? h_begin - a.heads[0] : h_begin / a.group;
  const int pos = a.next_pos != nullptr ? a.next_pos[s * a.n_kv_heads + unit] : a.positions != nullptr ? a.positions[row] : n;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    sn[i] = 0.f, cs[i] = 1.f;
    if (V * u + i < half) rotary_sincos(rot, V * u + i, pos, sn[i], cs[i]);
  }
  constexpr int UNROLL = 4;  // heads whose pieces are asked for before the first is used
  for (int h = h_begin; h < h_end; h += UNROLL) {
    Piece p0[UNROLL], p1[UNROLL];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i)
      if (h + i < h_end) {
        const int w = h + i >= a.heads[0] ? 1 : 0, hh = w ? h + i - a.heads[0] : h + i;
        const char* src = static_cast<const char*>(a.x[w]) + (s * a.in[w][0] + hh * a.in[w][1] + n * a.in[w][2]) * E;
        p0[i].load(src + c0 * E);
        if (second) p1[i].load(src + c1 * E);
      }
#pragma unroll
    for (int i = 0; i < UNROLL; ++i)
      if (h + i < h_end) {
        const int w = h + i >= a.heads[0] ? 1 : 0, hh = w ? h + i - a.heads[0] : h + i;
        rotary_turn<E, V, INTER>(p0[i], p1[i], sn, cs, u, half, turns);
        char* dst = static_cast<char*>(a.y[w]) + (s * a.out[w][0] + hh * a.out[w][1] + n * a.out[w][2]) * E;
        p0[i].store(dst + c0 * E);
        if (second) p1[i].store(dst + c1 * E);
      }
  }
}

}  // namespace he
