// Rotary positions (first_op_rope): pair i of a head turns by position * frequency i; the rest of the head passes unchanged.
//
//   (a, b) -> amplitude (a cos t - b sin t, a sin t + b cos t),  t = position * f_i;  transpose: sin -> -sin.
//
// Angles are formed in 64 bits (a position of 10^5 times a frequency of 1 has no digits to lose in 32), as turns, so that the
// reduction is one subtraction; sine and cosine of the rest in 32.
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

// grid (rows), a workgroup a row: the row's sines into LDS, then its heads.
template <typename T>
__global__ void __launch_bounds__(WG) k_rope(RopeArgs P) {
  __shared__ float2 cs[ROPE_MAX_PAIRS];
  const int half = P.rot / 2;
  for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
    __syncthreads();
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
