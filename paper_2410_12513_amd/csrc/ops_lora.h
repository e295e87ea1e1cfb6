// Projections with an adapter per row (first_op_gemm_nt_lora):
//   T[i][p] = scale[a_i] sum_k La[a_i][p][k] A[i][k],   C[i][j] (+)= sum_k A[i][k] W[j][k] + sum_p T[i][p] Lb[a_i][j][p]
// with a_i the adapter of row i; a_i outside [0, adapters): no second term.
#pragma once
#include "common.h"

namespace first {

constexpr int LORA_RMAX = 64;             // largest rank

struct LoraArgs {
  const void *A, *W, *La, *Lb;
  const int* adapter;
  const float* scale;
  float *C, *T;                           // T [m][rp] fp32, zero where there is no adapter and past the rank
  int m, n, k, r, rp, adapters, accumulate;
};

// T: grid (rows), a wave a rank.
template <typename E>
__global__ void __launch_bounds__(WG) k_lora_shrink(LoraArgs P) {
  const int row = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int a = P.adapter[row];
  const bool have = a >= 0 && a < P.adapters;
  const E* x = reinterpret_cast<const E*>(P.A) + (size_t)row * P.k;
  for (int p = wave; p < P.rp; p += WAVES) {
    float s = 0.f;
    if (have && p < P.r) {
      const E* w = reinterpret_cast<const E*>(P.La) + ((size_t)a * P.r + p) * P.k;
      for (int i = lane; i < P.k; i += 64) s = fmaf(to_f32(w[i]), to_f32(x[i]), s);
      s = wave_sum(s) * P.scale[a];
    }
    if (lane == 0) P.T[(size_t)row * P.rp + p] = s;
  }
}

// C: 64 x 64 tiles, 16 x 16 threads of 4 x 4 results.
template <typename E>
__global__ void __launch_bounds__(WG) k_lora_gemm(LoraArgs P) {
  __shared__ float a[16][65], w[16][65];
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < P.k; k0 += 16) {
    __syncthreads();
    for (int i = threadIdx.x; i < 1024; i += WG) {
      const int row = i >> 4, c = i & 15;
      const bool ok = k0 + c < P.k;
      a[c][row] = ok && m0 + row < P.m ? to_f32(reinterpret_cast<const E*>(P.A)[(size_t)(m0 + row) * P.k + k0 + c]) : 0.f;
      w[c][row] = ok && n0 + row < P.n ? to_f32(reinterpret_cast<const E*>(P.W)[(size_t)(n0 + row) * P.k + k0 + c]) : 0.f;
    }
    __syncthreads();
    for (int c = 0; c < 16; ++c)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[c][ty * 4 + i], w[c][tx * 4 + j], acc[i][j]);
  }
  for (int i = 0; i < 4; ++i) {
    const int row = m0 + ty * 4 + i;
    if (row >= P.m) continue;
    const int ad = P.adapter[row];
    for (int j = 0; j < 4; ++j) {
      const int col = n0 + tx * 4 + j;
      if (col >= P.n) continue;
      float s = acc[i][j];
      if (ad >= 0 && ad < P.adapters)
        for (int p = 0; p < P.r; ++p)
          s = fmaf(P.T[(size_t)row * P.rp + p], to_f32(reinterpret_cast<const E*>(P.Lb)[((size_t)ad * P.n + col) * P.r + p]), s);
      float* c = P.C + (size_t)row * P.n + col;
      *c = P.accumulate ? *c + s : s;
    }
  }
}

}  // namespace first
