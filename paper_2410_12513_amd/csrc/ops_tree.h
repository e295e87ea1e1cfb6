// Attention of trees of drafted tokens over the paged cache and over the trees themselves (first_op_tree_attn).
//   o = softmax(scale q K^T) V over the cached positions < len and the nodes that the node's mask names; 0 where there are none.
//
// The rows of a workgroup are (node, query head of one KV head) pairs of one sequence, so that the keys and values of a KV head are
// fetched once for all nodes and all of its query heads.  The keys are cut into splits; a workgroup walks one in tiles, with running maximum and
// sum, and where there are several splits a second kernel joins them.  Split 0 begins with the tree's own keys.
//
// us a call (in a trace: walk + join), 32 query heads on 8 of 128 dims, bf16, and what bounds it:
//   one node over 1000 positions        13.4 (10.4 + 3.2)  latency: offsets and lengths, keys, shares of a tile through LDS, the join
//   16 trees of 9 to 16 over 300-2300   31 (27.6 + 4.6)    loads, 89 MB at 3.2 TB/s in the walk, floor 17.5
//   4 trees of 33 to 61 over 20000 and more  157 (150 + 8.4)  matrix cores (without loads 130, loads alone 83), busy 43 % of the time: a third of the products are the weights'
//     second parts; floor 73
// Tried and slower or no faster: one workgroup a unit with a ring of four tiles (38 us in the second case), waves' priorities, an order of products and loads by hand,
// scores of the next tile formed between the exponentials of this one.
#pragma once
#include <type_traits>

#include "mfma_tiles.h"

namespace first {

struct TreeArgs {
  const void *q, *k, *v, *pool;           // q [N][Hq][hd]; k, v [N][Hkv][hd]; pool [page][K|V][Hkv][16][hd]
  const int *table, *lens, *offs;         // [B][max_pages], [B], [B + 1]
  const unsigned long long* mask;         // [N][words] or null: node i sees nodes 0 .. i
  void* out;
  float* lse;
  int B, N, Hq, Hkv, n_pages, max_pages, words, max_nodes, max_len;
  float scale;
  int split_keys, splits;                 // keys of a split, at least, and splits of max_len then
  int places, step, block;                // places > 0: the splits are as long as fills that many workgroups a KV head, a multiple of step; rows of a workgroup
  int* keys;                              // places > 0: how long they are, for the join
  float *part, *ml;                       // splits > 1: [split][N * Hq][hd] weighted values, [split][N * Hq][2] maximum (as an exponent of 2) and sum
};
constexpr int TREE_PAGE = 16, TREE_SPLIT_MAX = 8192;
constexpr int TREE_MAX_NODES = 2048;      // (a sequence's nodes through one descriptor: 2^11 nodes of 2^10 heads of 2^9 bytes)

// What the host and the kernels take of the numbers on the device.
struct TreeSeq { int o0, n, len; };
__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs& P, int b) {
  const int o0 = max(0, min(P.offs[b], P.N)), n = min(min(P.offs[b + 1], P.N) - o0, P.max_nodes);
  return {o0, max(n, 0), (int)max(0ll, min((long long)min(P.lens[b], P.max_len), (long long)P.max_pages * TREE_PAGE))};
}

// Keys of a split, B <= 64 sequences: the shortest multiple of step, not below split_keys, with which all workgroups that have any find a place at once.
__device__ __forceinline__ int tree_sums(int v) {          // running sum over the lanes
#define FIRST_SUM_STEP(CTRL, ROWS) v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
  FIRST_SUM_STEP(0x111, 0xf) FIRST_SUM_STEP(0x112, 0xf) FIRST_SUM_STEP(0x114, 0xf) FIRST_SUM_STEP(0x118, 0xf)
  FIRST_SUM_STEP(0x142, 0xa) FIRST_SUM_STEP(0x143, 0xc)
#undef FIRST_SUM_STEP
  return v;
}
// Which of them the nth workgroup of a KV head takes: those that have keys come first, one behind the other, as empty ones in between leave places to nobody.
struct TreeShare { int keys, b, split, rows; };            // b < 0: none
__device__ __forceinline__ TreeShare tree_share(const TreeArgs& P, int nth) {
  const int lane = threadIdx.x & 63;
  const TreeSeq q = tree_seq(P, min(lane, P.B - 1));
  const int blocks = lane < P.B ? (q.n * (P.Hq / P.Hkv) + P.block - 1) / P.block : 0, steps = (q.len + P.step - 1) / P.step, most = TREE_SPLIT_MAX / P.step;
  auto sum = [&](int v) { return __builtin_amdgcn_readlane(tree_sums(v), 63); };
  auto count = [&](int per) { return blocks * max(1, (steps + per - 1) / per); };
  // (what fits, to begin with; in 64ths and no more than 2^24 a sequence)
  int per = min(most, max(P.split_keys / P.step, sum((int)fminf((float)blocks * (float)steps / (float)P.places * 64.f, 16777216.f)) / 64));
  while (per < most && sum(count(per)) > P.places) per += max(1, per / 32);
  per = min(per, most);
  const int mine = count(per), through = tree_sums(mine);
  const unsigned long long past = __ballot(through > nth);
  if (past == 0) return {per * P.step, -1, 0, 0};
  const int b = __ffsll(past) - 1, rest = nth - (__builtin_amdgcn_readlane(through, b) - __builtin_amdgcn_readlane(mine, b)), rows = __builtin_amdgcn_readlane(blocks, b);
  return {per * P.step, b, rest / rows, rest % rows};
}

// 16 bytes of both operands, multiplied: 8 bf16 of each half of the wave in one product of depth 16, or 4 fp32 in four of depth 2.
__device__ __forceinline__ void tree_mma(bf16, floatx16_t& acc, u32x4_t a, u32x4_t b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void tree_mma(float, floatx16_t& acc, u32x4_t a, u32x4_t b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
}

// A tile of TK keys: rows of RB bytes, their 16-byte chunks permuted by row so that the reads below spread over all banks.  Keys are read a
// chunk of 32 rows at a time, values of four keys by 16 dims (bf16, transposed on the way), or of two keys by 32 dims (fp32).
template <int RB> __device__ __forceinline__ int tree_kslot(int row, int c) { return RB == 128 ? c ^ ((row >> 1) & 7) : c ^ (row & 15); }
template <typename E, int RB> __device__ __forceinline__ int tree_vslot(int row, int c) {
  if (sizeof(E) == 4) return c ^ (((row >> 2) & 1) * 8);
  return RB == 128 ? c ^ (((row >> 1) & 3) * 2) : c ^ ((row & 7) * 2);
}

typedef short tree_s4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) tree_s4_t* tree_lds4_t;

// QG groups of 32 rows x KH shares of a tile's keys (NS blocks of 32 each); S tiles in the ring.  grid (KV heads x blocks of 32 QG rows, splits, B);
// with places: (KV heads, places), what a workgroup takes by tree_share
//
// Everything is transposed, so that a lane owns ONE row of the result (column of the products): S^T = K Q^T and O^T = V^T P^T with the weights
// straight from the accumulators of S^T, bf16 ones split into two parts (with one part their rounding would be as large as that of the
// output).  The values' operand, eight keys of one dim, comes out of LDS through transposed reads.  Accumulators of the 32x32 MFMA: lane l
// holds column l % 32, register r holds row 8 (r / 4) + 4 (l / 32) + r % 4.
template <typename E, int HD, int QG, int KH, int NS, int S>
__global__ void __launch_bounds__(QG * KH * 64, QG == 1 ? 1 : 2) k_tree_attn(TreeArgs P) {
  constexpr int NW = QG * KH, TK = KH * NS * 32, RB = HD * (int)sizeof(E), CPR = RB / 16, RPL = 64 / CPR, NI = TK / RPL / NW;
  constexpr int KB = TK * RB, STG = 2 * KB, KS = RB / 32, DT = HD / 32;
  static_assert(TK % (RPL * NW) == 0 && NI >= 1 && TK % TREE_PAGE == 0, "whole loads");
  static_assert((size_t)QG * (KH - 1) * (16 * DT + 2) * 256 <= (size_t)S * STG, "partial results of the shares fit the ring");
  extern __shared__ __align__(16) char tree_smem[];
  __shared__ int pages[TREE_SPLIT_MAX / TREE_PAGE];
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)tree_smem;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 31, gl = lane >> 5;
  const int g = blockIdx.x % P.Hkv, G = P.Hq / P.Hkv;
  TreeShare mine = {P.split_keys, (int)blockIdx.z, (int)blockIdx.y, (int)blockIdx.x / P.Hkv};
  if (P.places > 0) {
    mine = tree_share(P, blockIdx.y);
    if ((blockIdx.x | blockIdx.y | threadIdx.x) == 0) *P.keys = mine.keys;
    if (mine.b < 0) return;
  }
  const int b = mine.b, split = mine.split, keys = mine.keys;
  const int row0 = mine.rows * (32 * QG), k_lo = split * keys;
  // the split's page ids before anybody knows how many of them count: one round trip less ahead of the first keys
  constexpr int PER = (TREE_SPLIT_MAX / TREE_PAGE + NW * 64 - 1) / (NW * 64);
  const int last_pg = min((k_lo + keys) / TREE_PAGE, P.max_pages) - 1;
  int ids[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int pg = k_lo / TREE_PAGE + (int)threadIdx.x + i * NW * 64;
    ids[i] = pg <= last_pg ? P.table[(size_t)b * P.max_pages + pg] : -1;
  }
  const TreeSeq q = tree_seq(P, b);
  const int rows = q.n * G, k_hi = min(q.len, k_lo + keys);
  if (row0 >= rows || (split > 0 && k_lo >= q.len)) return;
  const int n_tree = split == 0 ? (q.n + TK - 1) / TK : 0, n_tiles = n_tree + max(0, k_hi - k_lo + TK - 1) / TK;
  const int n_pg = max(0, k_hi - k_lo + TREE_PAGE - 1) / TREE_PAGE;
  bool hole = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int pg = (int)threadIdx.x + i * NW * 64;
    const bool ok = ids[i] >= 0 && ids[i] < P.n_pages;
    if (pg < n_pg) pages[pg] = ok ? ids[i] : -1;
    hole |= pg < n_pg && !ok;
  }
  const bool holes = __syncthreads_or(hole);

  const int qg = wave % QG, kh = wave / QG, ri = row0 + qg * 32 + col, rc = min(ri, rows - 1);
  const int node = rc / G, head = g * G + rc % G;
  const size_t orow = (size_t)(q.o0 + node) * P.Hq + head;
  const bool live = row0 + qg * 32 < rows;
  u32x4_t Q[KS];
  {
    const char* x = reinterpret_cast<const char*>(P.q) + orow * RB + gl * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      Q[s] = *reinterpret_cast<const u32x4_t*>(x + s * 32);
      if (P.scale < 0.f)                                   // (the sign goes to the queries: a maximum of scores is then one of exponents)
#pragma unroll
        for (int e = 0; e < 4; ++e) Q[s][e] ^= sizeof(E) == 2 ? 0x80008000u : 0x80000000u;
    }
  }
  // what this lane fetches of a tile's keys and values, and where that lies in a page
  const int lrow = lane / CPR;
  uint32_t ck[NI], cv[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int row = (wave * NI + i) * RPL + lrow;
    ck[i] = tree_kslot<RB>(row, lane % CPR) * 16;
    cv[i] = tree_vslot<E, RB>(row, lane % CPR) * 16;
  }
  const size_t page_bytes = (size_t)2 * P.Hkv * TREE_PAGE * RB;
  auto issue = [&](int t, int slot) __attribute__((always_inline)) {
    const uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds0 + (uint32_t)slot * STG + (uint32_t)wave * NI * 1024));
    if (t < n_tree) {
      const uint32_t pitch = (uint32_t)P.Hkv * RB, bytes = (uint32_t)(q.n - 1) * pitch + RB;
      const size_t first = ((size_t)q.o0 * P.Hkv + g) * RB;
      const i32x4_t rk = pg_rsrc(reinterpret_cast<const char*>(P.k) + first, bytes), rv = pg_rsrc(reinterpret_cast<const char*>(P.v) + first, bytes);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const uint32_t j = t * TK + (wave * NI + i) * RPL + lrow, off = j < (uint32_t)q.n ? j * pitch : 0x7ffffe00u;   // (no such node: zeros)
        pg_load_lds_any(at + i * 1024, off + ck[i], rk, 0u);
        pg_load_lds_any(at + KB + i * 1024, off + cv[i], rv, 0u);
      }
      return;
    }
    const int k0 = (t - n_tree) * TK;                      // from the split's first key
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = (wave * NI + i) * RPL, pg = (k0 + r) / TREE_PAGE, id = pg < n_pg ? __builtin_amdgcn_readfirstlane(pages[pg]) : -1;
      const i32x4_t rs = pg_rsrc(reinterpret_cast<const char*>(P.pool) + (size_t)max(id, 0) * page_bytes, id >= 0 ? (uint32_t)page_bytes : 0u);
      const uint32_t off = k_lo + k0 + r + lrow < k_hi ? (uint32_t)(g * TREE_PAGE + r % TREE_PAGE + lrow) * RB : 0x7ff00000u;   // (past the end: zeros)
      pg_load_lds_any(at + i * 1024, off + ck[i], rs, 0u);
      pg_load_lds_any(at + KB + i * 1024, off + (uint32_t)P.Hkv * TREE_PAGE * RB + cv[i], rs, 0u);
    }
  };

  floatx16_t O[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[t][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  const float sl = fmaxf(fabsf(P.scale) * LOG2E, 1.17549435e-38f);       // (never 0: that of a masked score stays -inf)
  // bits of the 32 nodes from j0 on that this lane's row sees, moved so that bit 8 (r / 4) + r % 4 is that of register r
  auto seen = [&](int j0) __attribute__((always_inline)) {
    const int left = q.n - j0;
    uint32_t w = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1u;
    if (left > 0) {
      if (P.mask != nullptr) w &= (uint32_t)(P.mask[(size_t)(q.o0 + node) * P.words + j0 / 64] >> (j0 % 64));
      else w &= node - j0 >= 31 ? ~0u : node < j0 ? 0u : (2u << (node - j0)) - 1u;
    }
    return w >> (4 * gl);
  };
  // One tile: n keys of it exist from the wave's first one on, k0 that key's number in the split or the tree.
  auto tile = [&](auto tree, const char* sk, int k0, int n) __attribute__((always_inline)) {
    const char* sv = sk + KB;
    floatx16_t W[NS];
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) W[u][r] = 0.f;
    {                                                      // (fragments requested in two halves ahead of the products: one by one, each product waited for its own)
      constexpr int H = sizeof(E) == 4 ? (NS == 2 ? 1 : 2) : NS == 2 ? 2 : KS / 2;
      u32x4_t kf[2][H][NS];
      auto fetch = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < H; ++s)
#pragma unroll
          for (int u = 0; u < NS; ++u) {
            const int row = (kh * NS + u) * 32 + col;
            kf[h & 1][s][u] = *reinterpret_cast<const u32x4_t*>(sk + row * RB + tree_kslot<RB>(row, 2 * (h * H + s) + gl) * 16);
          }
      };
      fetch(0);
#pragma unroll
      for (int h = 0; h < KS / H; ++h) {
        if (h + 1 < KS / H) fetch(h + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < H; ++s)
#pragma unroll
          for (int u = 0; u < NS; ++u) tree_mma(E{}, W[u], kf[h & 1][s][u], Q[h * H + s]);
      }
    }
    if (tree || n < NS * 32 || holes) {
#pragma unroll
      for (int u = 0; u < NS; ++u) {
        uint32_t w;
        if (tree) {
          w = seen(k0 + 32 * u);
        } else {
          const int left = n - 32 * u, pg = (k0 + 32 * u) / TREE_PAGE;
          w = left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1u;
          if (holes) w &= (pg < n_pg && pages[pg] >= 0 ? 0xffffu : 0u) | (pg + 1 < n_pg && pages[pg + 1] >= 0 ? 0xffff0000u : 0u);
          w >>= 4 * gl;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) W[u][r] = w >> (8 * (r >> 2) + (r & 3)) & 1u ? W[u][r] : -INFINITY;
      }
    }
    float mt = W[0][0];
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, W[u][r]);
    float ma, mb;
    both_halves(mt, ma, mb);
    // (the maximum as it enters the exponent, rounded once after its product: a weight is 2^(s sl - m) with one rounding of that difference)
    const float mn = fmaxf(m, fmaxf(ma, mb) * sl), mu = mn == -INFINITY ? 0.f : mn;      // (nothing seen yet: weights of 0)
    if (__any(mn > m)) {
      const float corr = __builtin_amdgcn_exp2f(m - mu);
      l *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] *= corr;
      m = mn;
    }
    float ls[4] = {0.f, 0.f, 0.f, 0.f};                    // the tile's sum first: a long cache's l is thousands of terms
#pragma unroll
    for (int u = 0; u < NS; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) { W[u][r] = __builtin_amdgcn_exp2f(fmaf(W[u][r], sl, -mu)); ls[r & 3] += W[u][r]; }
    l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
    if constexpr (sizeof(E) == 2) {
      // k-step s2 of a block: keys 16 s2 + 4 gl + 0..3 and 8 more, the rows of registers 8 s2 .. 8 s2 + 7
      auto values = [&](int s2) __attribute__((always_inline)) {
        union { uint32_t w[4]; u32x4_t x; } ph, pl;
        const int row = kh * NS * 32 + 16 * s2 + 4 * gl + ((lane & 15) >> 2);
        u32x4_t vf[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
          union { tree_s4_t s[2]; u32x4_t x; } f;
#pragma unroll
          for (int e = 0; e < 2; ++e)
            f.s[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tree_lds4_t)(sv + (row + 8 * e) * RB + tree_vslot<E, RB>(row + 8 * e, chunk) * 16 + (lane & 1) * 8));
          vf[d] = f.x;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) split_pair(W[s2 / 2][8 * (s2 & 1) + 2 * e], W[s2 / 2][8 * (s2 & 1) + 2 * e + 1], ph.w[e], pl.w[e]);
#pragma unroll
        for (int d = 0; d < DT; ++d) tree_mma(E{}, O[d], vf[d], pl.x);
#pragma unroll
        for (int d = 0; d < DT; ++d) tree_mma(E{}, O[d], vf[d], ph.x);
      };
#pragma unroll
      for (int s2 = 0; s2 < 2 * NS; ++s2) values(s2);
    } else {
#pragma unroll
      for (int u = 0; u < NS; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = (kh * NS + u) * 32 + 8 * (r >> 2) + 4 * gl + (r & 3);
#pragma unroll
          for (int d = 0; d < DT; ++d)
            O[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(sv + row * RB + tree_vslot<E, RB>(row, 8 * d + (col >> 2)) * 16 + (col & 3) * 4),
                                                        W[u][r], O[d], 0, 0, 0);
        }
    }
  };
  // The products take nodes that a row does not see times 0: an infinity or NaN there must not reach the row.  Where any is about (rare), the wave's share of
  // the tree again, a key at a time and only the seen ones.
  auto again = [&]() __attribute__((always_inline)) {
    bool odd = false;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) odd |= !(fabsf(O[d][r]) < INFINITY);
    if (!__any(odd)) return;
    m = -INFINITY; l = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[d][r] = 0.f;
    const E* qr = reinterpret_cast<const E*>(P.q) + orow * HD;
    const float sc = P.scale < 0.f ? -sl : sl;
    for (int j = 0; j < q.n; ++j) {
      if (j / (NS * 32) % KH != kh) continue;
      if (P.mask != nullptr ? !(P.mask[(size_t)(q.o0 + node) * P.words + j / 64] >> (j % 64) & 1) : j > node) continue;
      const size_t at = ((size_t)(q.o0 + j) * P.Hkv + g) * HD;
      const E *kr = reinterpret_cast<const E*>(P.k) + at, *vr = reinterpret_cast<const E*>(P.v) + at;
      float s = 0.f;
      for (int d = 0; d < HD; ++d) s = fmaf(to_f32(qr[d]), to_f32(kr[d]), s);
      s *= sc;
      const float top = fmaxf(m, s), use = top == -INFINITY ? 0.f : top, c = __builtin_amdgcn_exp2f(m - use), w = __builtin_amdgcn_exp2f(s - use);
      m = top;
      l = l * c + (gl == 0 ? w : 0.f);                     // (both halves of the wave hold the row, and add their sums at the end)
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] = fmaf(w, to_f32(vr[32 * d + 8 * (r >> 2) + 4 * gl + (r & 3)]), O[d][r] * c);
    }
  };

#pragma unroll
  for (int t = 0; t < S; ++t)
    if (t < n_tiles) issue(t, t);
  int slot = 0;
  auto arrived = [&](int t) __attribute__((always_inline)) {          // tile t is there; the tile S - 1 ahead goes where t - 1 was
    if (t == 0 && S <= n_tiles) pg_wait<2 * NI * (S - 1)>();
    else if (t > 0 && t + S - 2 < n_tiles) pg_wait<2 * NI * (S - 2)>();
    else pg_wait<0>();
    lds_barrier();
    if (t > 0 && t + S - 1 < n_tiles) issue(t + S - 1, slot == 0 ? S - 1 : slot - 1);
    const char* at = tree_smem + slot * STG;
    slot = slot + 1 == S ? 0 : slot + 1;
    return at;
  };
  int t = 0;
  for (; t < n_tree; ++t) {
    const char* at = arrived(t);
    const int k0 = t * TK + kh * NS * 32;
    if (live && k0 < q.n) tile(std::true_type{}, at, k0, q.n - k0);
  }
  if (live && n_tree > 0) again();
  for (; t < n_tiles; ++t) {
    const char* at = arrived(t);
    const int k0 = (t - n_tree) * TK + kh * NS * 32, n = k_hi - k_lo - k0;
    if (live && n > 0) tile(std::false_type{}, at, k0, n);
  }
  float la, lb;
  both_halves(l, la, lb);
  l = la + lb;
  if constexpr (KH > 1) {                                  // the shares of the keys meet in LDS
    float* ex = reinterpret_cast<float*>(tree_smem) + lane;
    constexpr int REC = (16 * DT + 2) * 64;
    lds_barrier();
    if (kh > 0) {
      float* to = ex + ((kh - 1) * QG + qg) * REC;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) to[(d * 16 + r) * 64] = O[d][r];
      to[16 * DT * 64] = m; to[(16 * DT + 1) * 64] = l;
    }
    lds_barrier();
    if (kh > 0) return;
#pragma unroll
    for (int w = 1; w < KH; ++w) {
      const float* from = ex + ((w - 1) * QG + qg) * REC;
      const float m2 = from[16 * DT * 64], l2 = from[(16 * DT + 1) * 64], top = fmaxf(m, m2), use = top == -INFINITY ? 0.f : top;
      const float c1 = __builtin_amdgcn_exp2f(m - use), c2 = __builtin_amdgcn_exp2f(m2 - use);
      m = top;
      l = l * c1 + l2 * c2;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] = O[d][r] * c1 + from[(d * 16 + r) * 64] * c2;
    }
  }
  if (ri >= rows) return;
  const bool whole = P.splits == 1;
  const float inv = !whole ? 1.f : l > 0.f || l != l ? 1.0f / l : 0.f;
  if (gl == 0) {
    if (!whole) *reinterpret_cast<float2*>(P.ml + ((size_t)split * P.N * P.Hq + orow) * 2) = make_float2(m, l);
    else if (P.lse != nullptr) P.lse[orow] = l == 0.f ? -INFINITY : (m + log2f(l)) * (1.f / LOG2E);
  }
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
      const int dim = 32 * d + 8 * rr + 4 * gl;
      const float4 o = make_float4(O[d][4 * rr] * inv, O[d][4 * rr + 1] * inv, O[d][4 * rr + 2] * inv, O[d][4 * rr + 3] * inv);
      if (!whole) *reinterpret_cast<float4*>(P.part + ((size_t)split * P.N * P.Hq + orow) * HD + dim) = o;
      else if constexpr (sizeof(E) == 2) *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(P.out) + orow * HD + dim) = make_uint2(pk_bf16(o.x, o.y), pk_bf16(o.z, o.w));
      else *reinterpret_cast<float4*>(reinterpret_cast<float*>(P.out) + orow * HD + dim) = o;
    }
}

// Joins the splits of a sequence: grid (rows / 4, B), a wave a row, lane: dims lane * HD / 64 ..  The splits of a row are those that have keys, and the first.
template <typename E, int HD>
__global__ void __launch_bounds__(WG) k_tree_join(TreeArgs P) {
  constexpr int DL = HD / 64;
  const int b = blockIdx.y, row = blockIdx.x * WAVES + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const TreeSeq q = tree_seq(P, b);
  if (row >= q.n * P.Hq) return;
  const size_t orow = (size_t)q.o0 * P.Hq + row, all = (size_t)P.N * P.Hq;
  const int keys = P.places > 0 ? *P.keys : P.split_keys, ns = max(1, (q.len + keys - 1) / keys);
  float M = -INFINITY, o[DL] = {}, L = 0.f;
  for (int s0 = 0; s0 < ns; s0 += 4) {                     // four splits requested together, and joined as they come
    float2 ml[4];
    float x[4][DL];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const size_t at = min(s0 + u, ns - 1) * all + orow;
      ml[u] = *reinterpret_cast<const float2*>(P.ml + at * 2);
#pragma unroll
      for (int e = 0; e < DL; ++e) x[u][e] = P.part[at * HD + lane * DL + e];
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < 4; ++u) top = fmaxf(top, ml[u].x);
    const float use = top == -INFINITY ? 0.f : top, c0 = __builtin_amdgcn_exp2f(M - use);
    M = top;
    L *= c0;
#pragma unroll
    for (int e = 0; e < DL; ++e) o[e] *= c0;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u < ns) {
        const float c = __builtin_amdgcn_exp2f(ml[u].x - use);
        L = fmaf(ml[u].y, c, L);
#pragma unroll
        for (int e = 0; e < DL; ++e) o[e] = fmaf(x[u][e], c, o[e]);
      }
  }
  const float inv = L > 0.f || L != L ? 1.0f / L : 0.f;
  E* out = reinterpret_cast<E*>(P.out) + orow * HD + lane * DL;
#pragma unroll
  for (int e = 0; e < DL; ++e) out[e] = from_f32<E>(o[e] * inv);
  if (lane == 0 && P.lse != nullptr) P.lse[orow] = L == 0.f ? -INFINITY : (M + log2f(L)) * (1.f / LOG2E);
}

}  // namespace first
