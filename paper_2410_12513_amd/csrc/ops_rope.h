// Rotary positions (first_op_rope): pair i of a head turns by position * frequency i; the rest of the head passes unchanged.
//
//   (a, b) -> amplitude (a cos t - b sin t, a sin t + b cos t),  t = position * f_i;  transpose: sin -> -sin.
//
// Angles are formed in 64 bits (a position of 10^5 times a frequency of 1 has no digits to lose in 32), as turns, so that the
// reduction is one subtraction; sine and cosine of the rest in 32.
//
// Bound: HBM, one read and one write of the heads; 16384 rows of 40 heads of 128 bf16 in 60 us, 5.6 TB/s.  (Pairs of elements a thread instead of chunks: 101 us.)  Small
// calls, 64 rows, 3.8 us: a round trip for the positions, the fp64 products, a round trip for the heads.
#pragma once
#include "common.h"

namespace first {

constexpr int ROPE_MAX_PAIRS = 128;       // head_dim <= 256

struct RopeArgs {
  const void* x;
  void* y;
  const int* positions;
  long long x_pitch, y_pitch;             // elements from a row to the next
  int rows, heads, hd, rot, interleaved;
  float amplitude, sign;
  double turns[ROPE_MAX_PAIRS];           // frequency / 2 pi
};

__device__ __forceinline__ float2 rope_cs(const RopeArgs& P, int pos, int i) {
  const double t = (double)pos * P.turns[i];
  const float f = (float)(t - rint(t));   // [-1/2, 1/2] turns
  float s, c;
  sincospif(2.f * f, &s, &c);
  return make_float2(c * P.amplitude, s * P.amplitude * P.sign);
}

// Rows whose heads start on 16 bytes and whose pairs fill whole chunks of 16 bytes: a workgroup takes R rows, their sines into LDS (a pair of a row a
// thread), then chunks of their heads: two of them, half a turned part apart (half), or one (interleaved) that hold whole pairs, or one that passes.
// ROPE_U chunks of a thread on their way at a time.
constexpr int ROPE_U = 4;
template <typename T, bool INTER, int R>
__global__ void __launch_bounds__(WG) k_rope_chunks(RopeArgs P) {
  constexpr int EPC = 16 / (int)sizeof(T), PAIRS = INTER ? EPC / 2 : EPC;
  __shared__ __align__(16) float2 cs[R * ROPE_MAX_PAIRS];
  const int half = P.rot / 2, turned = half / PAIRS, items = turned + (P.hd - P.rot) / EPC;      // of a head
  const long long row0 = (long long)blockIdx.x * R;
  const int rows = (int)min((long long)R, P.rows - row0);
  for (int i = threadIdx.x; i < rows * half; i += WG) cs[i] = rope_cs(P, P.positions[row0 + i / half], i % half);
  __syncthreads();
  const int total = rows * P.heads * items;
  const T* x0 = reinterpret_cast<const T*>(P.x) + row0 * P.x_pitch;
  T* y0 = reinterpret_cast<T*>(P.y) + row0 * P.y_pitch;
  for (int j0 = threadIdx.x; j0 < total; j0 += ROPE_U * WG) {
    u32x4_t a[ROPE_U], b[ROPE_U];
    int row[ROPE_U], at[ROPE_U], c[ROPE_U];
#pragma unroll
    for (int u = 0; u < ROPE_U; ++u) {
      const int j = min(j0 + u * WG, total - 1), h = j / items;
      c[u] = j - h * items;
      row[u] = h / P.heads;
      at[u] = (h - row[u] * P.heads) * P.hd + (c[u] < turned ? c[u] * EPC : P.rot + (c[u] - turned) * EPC);
      const T* x = x0 + row[u] * P.x_pitch + at[u];
      a[u] = *reinterpret_cast<const u32x4_t*>(x);
      if (!INTER) b[u] = *reinterpret_cast<const u32x4_t*>(x + (c[u] < turned ? half : 0));
    }
#pragma unroll
    for (int u = 0; u < ROPE_U; ++u) {
      if (j0 + u * WG >= total) break;
      T* y = y0 + row[u] * P.y_pitch + at[u];
      if (c[u] >= turned) {
        *reinterpret_cast<u32x4_t*>(y) = a[u];
        continue;
      }
      const float2* w = cs + row[u] * half + c[u] * PAIRS;
      float v[2 * PAIRS], o[2 * PAIRS];                    // half: the first elements, then the second; interleaved: as they stand
      auto widen = [&](u32x4_t r, float* to) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 2) { to[2 * e] = __uint_as_float(r[e] << 16); to[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u); }
          else to[e] = __uint_as_float(r[e]);
        }
      };
      widen(a[u], v);
      if (!INTER) widen(b[u], v + EPC);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const int ia = INTER ? 2 * i : i, ib = INTER ? 2 * i + 1 : i + PAIRS;
        const float2 t = w[i];
        o[ia] = v[ia] * t.x - v[ib] * t.y;
        o[ib] = v[ia] * t.y + v[ib] * t.x;
      }
      auto narrow = [&](const float* from) __attribute__((always_inline)) {
        u32x4_t r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = sizeof(T) == 2 ? pk_bf16(from[2 * e], from[2 * e + 1]) : __float_as_uint(from[e]);
        return r;
      };
      *reinterpret_cast<u32x4_t*>(y) = narrow(o);
      if (!INTER) *reinterpret_cast<u32x4_t*>(y + half) = narrow(o + EPC);
    }
  }
}

// Any other row (odd pitches and offsets, pairs that fill no chunk): grid (rows), a workgroup a row, an element pair a thread.
template <typename T>
__global__ void __launch_bounds__(WG) k_rope(RopeArgs P) {
  __shared__ float2 cs[ROPE_MAX_PAIRS];
  const int half = P.rot / 2;
  {
    const long long row = blockIdx.x;
    for (int i = threadIdx.x; i < half; i += WG) cs[i] = rope_cs(P, P.positions[row], i);
    __syncthreads();
    const T* x = reinterpret_cast<const T*>(P.x) + row * P.x_pitch;
    T* y = reinterpret_cast<T*>(P.y) + row * P.y_pitch;
    for (int j = threadIdx.x; j < P.heads * (P.hd - half); j += WG) {
      const int h = j / (P.hd - half), i = j - h * (P.hd - half);
      const T* xh = x + (size_t)h * P.hd;
      T* yh = y + (size_t)h * P.hd;
      if (i < half) {
        const int ia = P.interleaved ? 2 * i : i, ib = P.interleaved ? 2 * i + 1 : i + half;
        const float a = to_f32(xh[ia]), b = to_f32(xh[ib]);
        const float2 w = cs[i];
        yh[ia] = from_f32<T>(a * w.x - b * w.y);
        yh[ib] = from_f32<T>(a * w.y + b * w.x);
      } else {
        yh[i + half] = xh[i + half];
      }
    }
  }
}

}  // namespace first
