// Attention of trees of drafted tokens over the paged cache and over the trees themselves (first_op_tree_attn).
//   o = softmax(scale q K^T) V over the cached positions < len and the nodes that the node's mask names; 0 where there are none.
#pragma once
#include "common.h"

namespace first {

struct TreeArgs {
  const void *q, *k, *v, *pool;           // q [N][Hq][hd]; k, v [N][Hkv][hd]; pool [page][K|V][Hkv][16][hd]
  const int *table, *lens, *offs;         // [B][max_pages], [B], [B + 1]
  const unsigned long long* mask;         // [N][words] or null: node i sees nodes 0 .. i
  void* out;
  float* lse;
  int B, N, Hq, Hkv, n_pages, max_pages, words, max_nodes, max_len;
  float scale;
};
constexpr int TREE_PAGE = 16;

// grid (nodes, query heads, sequences): a workgroup a row, a wave every fourth key.
template <typename E, int HD>
__global__ void __launch_bounds__(WG) k_tree_rows(TreeArgs P) {
  __shared__ float red[WAVES][HD + 2];
  constexpr int DL = HD / 64;
  const int b = blockIdx.z, h = blockIdx.y, i = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int o0 = max(0, min(P.offs[b], P.N)), n = min(min(P.offs[b + 1], P.N) - o0, P.max_nodes);
  if (i >= n) return;
  const int len = max(0, min(min(P.lens[b], P.max_len), P.max_pages * TREE_PAGE)), g = h / (P.Hq / P.Hkv);
  const size_t page = (size_t)2 * P.Hkv * TREE_PAGE * HD;
  float q[DL], o[DL] = {}, m = -INFINITY, l = 0.f;
  for (int e = 0; e < DL; ++e) q[e] = to_f32(reinterpret_cast<const E*>(P.q)[((size_t)(o0 + i) * P.Hq + h) * HD + lane * DL + e]);
  auto take = [&](const E* kr, const E* vr) {
    float s = 0.f;
    for (int e = 0; e < DL; ++e) s = fmaf(q[e], to_f32(kr[lane * DL + e]), s);
    s = wave_sum(s) * P.scale;
    const float mn = fmaxf(m, s), c = m == -INFINITY ? 0.f : expf(m - mn), w = expf(s - mn);
    l = l * c + w;
    m = mn;
    for (int e = 0; e < DL; ++e) o[e] = o[e] * c + w * to_f32(vr[lane * DL + e]);
  };
  for (int j = wave; j < len; j += WAVES) {
    const int id = P.table[(size_t)b * P.max_pages + j / TREE_PAGE];
    if (id < 0 || id >= P.n_pages) continue;
    const E* kr = reinterpret_cast<const E*>(P.pool) + (size_t)id * page + ((size_t)g * TREE_PAGE + j % TREE_PAGE) * HD;
    take(kr, kr + (size_t)P.Hkv * TREE_PAGE * HD);
  }
  for (int j = wave; j < n; j += WAVES) {
    if (P.mask ? !(P.mask[(size_t)(o0 + i) * P.words + j / 64] >> (j % 64) & 1) : j > i) continue;
    const size_t at = ((size_t)(o0 + j) * P.Hkv + g) * HD;
    take(reinterpret_cast<const E*>(P.k) + at, reinterpret_cast<const E*>(P.v) + at);
  }
  for (int e = 0; e < DL; ++e) red[wave][lane * DL + e] = o[e];
  if (lane == 0) { red[wave][HD] = m; red[wave][HD + 1] = l; }
  __syncthreads();
  float M = -INFINITY, L = 0.f;
  for (int w = 0; w < WAVES; ++w) M = fmaxf(M, red[w][HD]);
  for (int w = 0; w < WAVES; ++w) L += red[w][HD + 1] > 0.f ? red[w][HD + 1] * expf(red[w][HD] - M) : 0.f;
  for (int d = threadIdx.x; d < HD; d += WG) {
    float s = 0.f;
    for (int w = 0; w < WAVES; ++w)
      if (red[w][HD + 1] > 0.f) s += red[w][d] * expf(red[w][HD] - M);
    reinterpret_cast<E*>(P.out)[((size_t)(o0 + i) * P.Hq + h) * HD + d] = from_f32<E>(L > 0.f ? s / L : 0.f);
  }
  if (threadIdx.x == 0 && P.lse) P.lse[(size_t)(o0 + i) * P.Hq + h] = L > 0.f ? M + logf(L) : -INFINITY;
}

}  // namespace first
