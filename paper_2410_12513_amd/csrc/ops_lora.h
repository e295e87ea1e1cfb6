// Projections with an adapter per row (first_op_gemm_nt_lora):
//   T[i][p] = scale[a_i] sum_k La[a_i][p][k] A[i][k],   C[i][j] (+)= sum_k A[i][k] W[j][k] + sum_p T[i][p] Lb[a_i][j][p]
// with a_i the adapter of row i; a_i outside [0, adapters): no second term.
//
// Few rows (decode steps): one pass over W, bound by its bytes.  k_lora_stream cuts W into 64 rows x a slice of K a workgroup, enough of
// them to keep the whole chip loading, and forms T beside it; k_lora_finish adds the slices and the adapters' second products.
//   16 x 4096 x 4096, rank 8, 16 adapters, bf16: 16 us a call (13.1 + 4.3 in a trace), 36 MB at 2.2 TB/s, floor 7.1: a launch's start and end and the join are half of it.
// More rows: T first (k_lora_shrink), then k_lora_tile, tiles through LDS with the second product ahead of the first K step; or, where a few tiles would leave
// the chip idle, tiles of slices of K and k_lora_finish.
//   250 x 14336 x 4096, rank 16: 55 us (48 tiles + 10 T), floor 27; a compute unit's loads arrive at 60 bytes a ns, 470 MB of them in 128 x 128 tiles.
//   4096 x 4096 x 14336, rank 8: 435 us (400-430 tiles + 50 T), 1.11 PFLOP/s, floor 341 at the rate of a large product; loads alone take 380: L2 delivers rows
//   28 KB apart at half of its rate for adjacent ones.  Matrix cores are busy 63 % of the time.
//
// Products of bf16 values are exact in fp32, and T stays fp32: three bf16 parts in its product.  A product with an adapter is kept apart and
// added to its own rows only, so an infinity in an adapter stays with the rows that use it.
#pragma once
#include "mfma_tiles.h"

namespace first {

constexpr int LORA_RMAX = 64;             // largest rank
constexpr int LORA_STREAM_ROWS = 64;

struct LoraArgs {
  const void *A, *W, *La, *Lb;
  const int* adapter;
  const float* scale;
  float *C, *T;                           // T [m][rp] fp32, zero where there is no adapter and past the rank
  float* part;                            // [ks][m][n] fp32, slices of K
  int m, n, k, r, rp, adapters, accumulate;
  int ks, gm, gn, shrink_tiles, shrink_ways;   // slices of K; row and column tiles; workgroups that form T: 16-row tiles x ways
};

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4_t;
__device__ __forceinline__ int lora_uni(int v) { return __builtin_amdgcn_readfirstlane(v); }
// a chunk of 16 bytes of a row of A and of one of W: lane = row + 32 half (32x32), row + 16 quarter (16x16)
__device__ __forceinline__ void lora_mma32(bf16, floatx16_t& acc, u32x4_t a, u32x4_t b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void lora_mma32(float, floatx16_t& acc, u32x4_t a, u32x4_t b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
}
__device__ __forceinline__ void lora_mma16(bf16, floatx4_t& acc, u32x4_t a, u32x4_t b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void lora_mma16(float, floatx4_t& acc, u32x4_t a, u32x4_t b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
}
// place of a row's 16-byte chunk in LDS: rows of 128 bytes (two rows are all banks), and of 64 (four are)
template <int RB> __device__ __forceinline__ int lora_slot(int row, int c) { return RB == 128 ? c ^ ((row >> 1) & 7) : c ^ ((row >> 2) & 3); }

// Ranks p0 .. of a row of Lb that begins at element `at`, a chunk of them; zeros from rank r on, whatever stands there (the next row: not multiplied even
// by 0).  One load where the chunk lies inside the array (rows of odd ranks begin anywhere; loads from global memory need no alignment), else one by one.
template <typename E> __device__ __forceinline__ u32x4_t lora_ranks(const E* lb, size_t at, size_t total, int p0, int r) {
  constexpr int EPC = 16 / (int)sizeof(E);
  union { E e[EPC]; u32x4_t v; } f;
  f.v = u32x4_t{0, 0, 0, 0};
  const int left = r - p0;
  if (left <= 0) return f.v;
  if (at + p0 + EPC <= total) {
    __builtin_memcpy(&f.v, lb + at + p0, 16);
    if (left < EPC)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        constexpr int PER = 4 / (int)sizeof(E);            // elements of a word
        const int n = left - d * PER;
        f.v[d] = n >= PER ? f.v[d] : n <= 0 ? 0u : f.v[d] & 0xffffu;
      }
    return f.v;
  }
#pragma unroll
  for (int e = 0; e < EPC; ++e)
    if (e < left) f.e[e] = lb[at + p0 + e];
  return f.v;
}

// ---- T ---------------------------------------------------------------------------------------------------------------------
// A workgroup takes 16 rows and every ways-th of the adapters among them; its waves share K out in steps of 128 bytes a row, and their sums meet in LDS.
// Rows without an adapter get their zeros from way 0.  red: NW * 16 * rp floats.
template <typename E, int NW, int NP>     // NP: blocks of 16 ranks, all of them (rp = 16 NP)
__device__ __forceinline__ void lora_shrink(const LoraArgs& P, int tile, int way, float* red) {
  constexpr int EPC = 16 / (int)sizeof(E), RP = 16 * NP;   // elements of a chunk
  constexpr int U = NP == 1 ? 8 : NP == 2 ? 4 : 2;         // half steps of a wave requested together
  const int wave = lora_uni((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, row = lane & 15, quarter = lane >> 4;
  const int m0 = tile * 16, mr = min(m0 + row, P.m - 1);
  const int id = P.adapter[mr];
  const bool have = m0 + row < P.m && id >= 0 && id < P.adapters;
  if (way == 0)
    for (int i = threadIdx.x; i < 16 * RP; i += NW * 64) {
      const int at = min(m0 + i / RP, P.m - 1), a = P.adapter[at];
      if (m0 + i / RP < P.m && (a < 0 || a >= P.adapters)) P.T[(size_t)at * RP + i % RP] = 0.f;
    }
  unsigned long long todo = __ballot(have) & 0xffffull;
  const int steps = (P.k + 8 * EPC - 1) / (8 * EPC);
  const E* x = reinterpret_cast<const E*>(P.A) + (size_t)mr * P.k;
  for (int nth = 0; todo != 0; ++nth) {
    const int a = __builtin_amdgcn_readlane(id, __ffsll(todo) - 1);
    const unsigned long long mine = __ballot(have && id == a) & 0xffffull;
    todo &= ~mine;
    if (nth % P.shrink_ways != way) continue;
    floatx4_t acc[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) acc[p] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    const E* la = reinterpret_cast<const E*>(P.La) + (size_t)a * P.r * P.k;
    for (int s0 = wave; s0 < steps; s0 += U / 2 * NW) {
      u32x4_t xa[U], w[U][NP];
#pragma unroll
      for (int u = 0; u < U; ++u) {                        // (both halves of a line by the same wave)
        const int at = (s0 + u / 2 * NW) * 8 * EPC + (2 * quarter + u % 2) * EPC;
        const bool ok = at < P.k;
        xa[u] = ok ? *reinterpret_cast<const u32x4_t*>(x + at) : u32x4_t{0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < NP; ++p) w[u][p] = ok && 16 * p + row < P.r ? *reinterpret_cast<const u32x4_t*>(la + (size_t)(16 * p + row) * P.k + at) : u32x4_t{0, 0, 0, 0};
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int p = 0; p < NP; ++p) lora_mma16(E{}, acc[p], xa[u], w[u][p]);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < NP; ++p)                           // lane: rank 16 p + lane % 16 of rows 4 (lane / 16) ..
#pragma unroll
      for (int e = 0; e < 4; ++e) red[(wave * 16 + 4 * quarter + e) * RP + 16 * p + row] = acc[p][e];
    __syncthreads();
    const float s = P.scale[a];
    for (int i = threadIdx.x; i < 16 * RP; i += NW * 64) {
      const int rr = i / RP;
      if (!(mine >> rr & 1)) continue;
      float t = 0.f;
      for (int w = 0; w < NW; ++w) t += red[w * 16 * RP + i];
      P.T[(size_t)(m0 + rr) * RP + i % RP] = i % RP < P.r ? t * s : 0.f;
    }
  }
}
template <typename E, int NW> __device__ __forceinline__ void lora_shrink(const LoraArgs& P, int at, float* red) {
  const int tile = at % P.shrink_tiles, way = at / P.shrink_tiles;
  if (P.rp == 16) lora_shrink<E, NW, 1>(P, tile, way, red);
  else if (P.rp == 32) lora_shrink<E, NW, 2>(P, tile, way, red);
  else lora_shrink<E, NW, 4>(P, tile, way, red);
}
constexpr int LORA_SHRINK_WAVES = 16;
template <typename E> __global__ void __launch_bounds__(LORA_SHRINK_WAVES * 64) k_lora_shrink(LoraArgs P) {
  extern __shared__ __align__(16) char lora_smem[];
  lora_shrink<E, LORA_SHRINK_WAVES>(P, blockIdx.x, reinterpret_cast<float*>(lora_smem));
}

// ---- few rows --------------------------------------------------------------------------------------------------------------
// The first shrink_tiles * shrink_ways workgroups form T; the others take 64 rows of W (a wave 16) x a slice of K.  The slice of A goes into LDS once, and
// every wave loads its rows of W straight into a ring of its own: it waits for nobody.  Two workgroups a compute unit (80 KB each), up to 80 KB of W in
// flight on it (five of a wave's six steps).  Partial sums [slice][m][n].
constexpr int LORA_A_BYTES = 32 * 1024;   // of LDS for the slice of A
template <typename E, int MR, int S>      // MR: 16, 32 or 64 rows of A; S steps in a wave's ring
__global__ void __launch_bounds__(WG, 2) k_lora_stream(LoraArgs P) {
  constexpr int RB = 128, EPS = RB / (int)sizeof(E), STG = 16 * RB;
  extern __shared__ __align__(16) char lora_smem[];
  const int helpers = P.shrink_tiles * P.shrink_ways;
  if ((int)blockIdx.x < helpers) {
    lora_shrink<E, WAVES>(P, blockIdx.x, reinterpret_cast<float*>(lora_smem));
    return;
  }
  const int id = blockIdx.x - helpers, wave = lora_uni((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, row = lane & 15, quarter = lane >> 4;
  const int slice = id % P.ks, n0 = (id / P.ks) * 64 + wave * 16;
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)lora_smem, ring0 = lds0 + LORA_A_BYTES + wave * S * STG;
  const char* ring = lora_smem + LORA_A_BYTES + wave * S * STG;
  const uint32_t pitch = (uint32_t)P.k * sizeof(E);
  const int rows_w = max(0, min(16, P.n - n0));
  const i32x4_t rw = pg_rsrc(reinterpret_cast<const char*>(P.W) + (size_t)min(n0, P.n - 1) * pitch, rows_w * pitch);
  const i32x4_t ra = pg_rsrc(P.A, P.m * pitch);
  const int steps = (P.k + EPS - 1) / EPS, s0 = (int)((long long)steps * slice / P.ks), s1 = (int)((long long)steps * (slice + 1) / P.ks);
  const int tail = (int)(pitch % RB) / 16;                 // chunks of the last step that exist (0: all)
  const int lrow = lane >> 3, lch = lane & 7;
  auto fetch = [&](uint32_t to, i32x4_t rs, int r, int s) __attribute__((always_inline)) {       // rows r .. r + 7 of step s
    const int chunk = lora_slot<RB>(r + lrow, lch);
    const uint32_t off = tail != 0 && s == steps - 1 && chunk >= tail ? 0x7ffffff0u : (uint32_t)(r + lrow) * pitch + chunk * 16;
    pg_load_lds_any((uint32_t)lora_uni((int)to), off, rs, (uint32_t)lora_uni(s * RB));
  };
  for (int i = wave; i < (s1 - s0) * (MR / 8); i += WAVES) fetch(lds0 + i * 1024, ra, i % (MR / 8) * 8, s0 + i / (MR / 8));
  auto issue = [&](int s, int slot) __attribute__((always_inline)) {
    fetch(ring0 + slot * STG, rw, 0, s);
    fetch(ring0 + slot * STG + 1024, rw, 8, s);
  };
  floatx4_t acc[MR / 16];
#pragma unroll
  for (int i = 0; i < MR / 16; ++i) acc[i] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < S - 1; ++s)
    if (s0 + s < s1) issue(s0 + s, s);
  if (s1 - s0 >= S - 1) pg_wait<2 * (S - 1)>(); else pg_wait<0>();      // (A is older)
  lds_barrier();
  int slot = 0;
  for (int s = s0; s < s1; ++s) {
    // (the slot that is loaded into was read a step ago: its reads have ended, the products took their results)
    if (s + S - 1 < s1) { issue(s + S - 1, slot == 0 ? S - 1 : slot - 1); pg_wait<2 * (S - 1)>(); } else { pg_wait<0>(); }
    const char *at = ring + slot * STG, *xa = lora_smem + (s - s0) * MR * RB;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const u32x4_t w = *reinterpret_cast<const u32x4_t*>(at + row * RB + lora_slot<RB>(row, 4 * c + quarter) * 16);
#pragma unroll
      for (int i = 0; i < MR / 16; ++i)
        lora_mma16(E{}, acc[i], *reinterpret_cast<const u32x4_t*>(xa + (16 * i + row) * RB + lora_slot<RB>(16 * i + row, 4 * c + quarter) * 16), w);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    slot = slot + 1 == S ? 0 : slot + 1;
  }
  if (n0 + row < P.n) {
    float* to = P.part + (size_t)slice * P.m * P.n + n0 + row;
#pragma unroll
    for (int i = 0; i < MR / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (16 * i + 4 * quarter + e < P.m) to[(size_t)(16 * i + 4 * quarter + e) * P.n] = acc[i][e];
  }
}

// C from the slices of K, the adapters' second products and what was there: grid (columns / 256, rows).  Bound by two round trips: the row's adapter, then everything else.
template <typename E>
__global__ void __launch_bounds__(WG) k_lora_finish(LoraArgs P) {
  constexpr int EPC = 16 / (int)sizeof(E);
  const int row = blockIdx.y, col = blockIdx.x * WG + threadIdx.x;
  if (col >= P.n) return;
  const int a = P.adapter[row];
  float* const c = P.C + (size_t)row * P.n + col;
  float s = 0.f;
  for (int u = 0; u < P.ks; ++u) s += P.part[((size_t)u * P.m + row) * P.n + col];
  if (a >= 0 && a < P.adapters) {
    const float* t = P.T + (size_t)row * P.rp;
    const size_t at = ((size_t)a * P.n + col) * P.r, all = (size_t)P.adapters * P.n * P.r;
    float d = 0.f;
    for (int p = 0; p < P.r; p += EPC) {
      union { u32x4_t v; E e[EPC]; } w = {lora_ranks(reinterpret_cast<const E*>(P.Lb), at, all, p, P.r)};
#pragma unroll
      for (int e = 0; e < EPC; ++e) d = fmaf(t[p + e], to_f32(w.e[e]), d);
    }
    s += d;
  }
  *c = P.accumulate ? *c + s : s;
}

// ---- more rows -------------------------------------------------------------------------------------------------------------
// BM x BN tile, WGM x WGN waves, K steps of RB bytes a row, S of them in the LDS ring; loads go straight into LDS, a row's chunks permuted against bank
// conflicts (none counted), and the fragments of the next 32 bytes of K are read while the present ones are multiplied, across the barrier too.  ks > 1: partial sums
// of a slice of K; ks = 1: the adapters' second products and the result.  Accumulators of the 32x32 MFMA: lane l holds column l % 32, register r holds
// row 8 (r / 4) + 4 (l / 32) + r % 4.
//   256 x 256: steps of 128 bytes, two of them in LDS; of 64 bytes, four of them, half a line a load: 490 us against 437 at 4096 x 4096 x 14336.  Four waves of 128 x 128: 557.
//   Requesting the lines of later steps into L2 ahead of time made it slower (444 -> 467; 60 -> 71 at 250 x 14336 x 4096).
template <typename E, int BM, int BN, int WGM, int WGN, int RB, int S>
__global__ void __launch_bounds__(WGM * WGN * 64, 1) k_lora_tile(LoraArgs P) {
  constexpr int NW = WGM * WGN, TM = BM / WGM, TN = BN / WGN, IM = TM / 32, JN = TN / 32, EPC = 16 / (int)sizeof(E);
  constexpr int RPL = 1024 / RB, CPR = RB / 16, IA = BM / RPL / NW, IB = BN / RPL / NW, NL = IA + IB, STG = (BM + BN) * RB, NKK = RB / 32;
  static_assert(BM % (RPL * NW) == 0 && BN % (RPL * NW) == 0 && TM % 32 == 0 && TN % 32 == 0 && (TM <= 64 || TM == 128), "tile shape");
  extern __shared__ __align__(16) char lora_smem[];
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)lora_smem;
  const int wave = lora_uni((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, lr = lane & 31, lg = lane >> 5;
  // Workgroup -> tile: consecutive workgroups go to the eight XCDs in turn; each gets a contiguous run of tiles, in groups of a few row tiles with the row
  // tiles of a column next to each other, so that what runs on an XCD at a time is a compact block of tiles whose operands its L2 holds.
  int id = blockIdx.x;
  {
    const int total = gridDim.x, per = total / 8, rem = total % 8, x = id % 8;
    id = x * per + min(x, rem) + id / 8;
  }
  const int slice = id % P.ks;
  id /= P.ks;
  constexpr int GR = BM == 256 ? 4 : 8;
  const int grp = id / (GR * P.gn), in = id - grp * GR * P.gn, grn = min(GR, P.gm - grp * GR);
  const int m0 = (grp * GR + in % grn) * BM, n0 = (in / grn) * BN;
  const uint32_t pitch = (uint32_t)P.k * sizeof(E);
  const int rowsA = min(BM, P.m - m0), rowsB = min(BN, P.n - n0);
  const i32x4_t ra = pg_rsrc(reinterpret_cast<const char*>(P.A) + (size_t)m0 * pitch, rowsA * pitch);
  const i32x4_t rb = pg_rsrc(reinterpret_cast<const char*>(P.W) + (size_t)n0 * pitch, rowsB * pitch);
  const int nsteps = (int)((pitch + RB - 1) / RB), tail = (int)(pitch % RB) / 16;
  const int s0 = (int)((long long)nsteps * slice / P.ks), s1 = (int)((long long)nsteps * (slice + 1) / P.ks);
  // Workgroups of an XCD walk K from the same place, those of different ones from different places: 60 us -> 56 at 250 x 14336 x 4096, where all of them asked for the
  // same columns of 14336 rows at a time.
  const int rot = s1 > s0 ? (int)(blockIdx.x % 8) * 5 % (s1 - s0) : 0;
  uint32_t va[IA], vb[IB];
  const int lrow = lane / CPR, lch = lane % CPR;
#pragma unroll
  for (int i = 0; i < IA; ++i) { const int r = (wave * IA + i) * RPL + lrow; va[i] = r * pitch + lora_slot<RB>(r, lch) * 16; }
#pragma unroll
  for (int i = 0; i < IB; ++i) { const int r = (wave * IB + i) * RPL + lrow; vb[i] = r * pitch + lora_slot<RB>(r, lch) * 16; }
  auto issue = [&](int step, int slot) __attribute__((always_inline)) {
    step = step + rot < s1 ? step + rot : step + rot - (s1 - s0);
    const uint32_t b = (uint32_t)lora_uni((int)(lds0 + (uint32_t)slot * STG)), so = (uint32_t)lora_uni(step * RB);
    const bool cut = tail != 0 && step == nsteps - 1;
    auto off = [&](uint32_t v, int r) __attribute__((always_inline)) { return cut && lora_slot<RB>(r, lch) >= tail ? 0x7ffffff0u : v; };   // (past the row's end: zeros)
#pragma unroll
    for (int i = 0; i < IA; ++i) pg_load_lds_any(b + (wave * IA + i) * 1024, off(va[i], (wave * IA + i) * RPL + lrow), ra, so);
#pragma unroll
    for (int i = 0; i < IB; ++i) pg_load_lds_any(b + BM * RB + (wave * IB + i) * 1024, off(vb[i], (wave * IB + i) * RPL + lrow), rb, so);
  };
  floatx16_t acc[IM][JN];
#pragma unroll
  for (int i = 0; i < IM; ++i)
#pragma unroll
    for (int j = 0; j < JN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const int wm = (wave / WGN) * TM, wn = (wave % WGN) * TN;
  uint32_t oa[NKK], ob[NKK];
#pragma unroll
  for (int k = 0; k < NKK; ++k) {
    oa[k] = (wm + lr) * RB + lora_slot<RB>(wm + lr, 2 * k + lg) * 16;
    ob[k] = BM * RB + (wn + lr) * RB + lora_slot<RB>(wn + lr, 2 * k + lg) * 16;
  }
  u32x4_t fa[2][IM], fb[2][JN];
  auto frags = [&](int buf, int slot, int k) __attribute__((always_inline)) {
    const char* base = lora_smem + slot * STG;
#pragma unroll
    for (int j = 0; j < JN; ++j) fb[buf][j] = *reinterpret_cast<const u32x4_t*>(base + ob[k] + j * 32 * RB);
#pragma unroll
    for (int i = 0; i < IM; ++i) fa[buf][i] = *reinterpret_cast<const u32x4_t*>(base + oa[k] + i * 32 * RB);
  };
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (s0 + s < s1) issue(s0 + s, s);

  if (P.ks == 1) {
    // The second product first, while the first tiles are on their way: for 64 of this wave's rows at a time the adapters among them, one after the other, in steps of
    // two chunks of ranks.  What a step needs is requested while the one before it is multiplied: rows of many adapters were as many round trips in a row.
    constexpr int H = IM < 2 ? IM : 2;
    struct Step { unsigned long long rows; u32x4_t w[JN], t[H][EPC / 4]; };
#pragma unroll
    for (int h = 0; h < IM / H; ++h) {
      const int mine = m0 + wm + 64 * h + min(lane, TM - 1), ad = P.adapter[min(mine, P.m - 1)];
      unsigned long long todo = __ballot(lane < TM && mine < P.m && ad >= 0 && ad < P.adapters), rows = 0;
      int a = 0, p = P.r;
      auto next = [&](Step& st) __attribute__((always_inline)) {
        if (p >= P.r) {                                    // the next adapter
          if (todo == 0) return false;
          a = __builtin_amdgcn_readlane(ad, __ffsll(todo) - 1);
          rows = __ballot(ad == a) & todo;
          todo &= ~rows;
          p = 0;
        }
        st.rows = rows;
        const int p0 = p + lg * EPC;
        const E* const lb = reinterpret_cast<const E*>(P.Lb);
#pragma unroll
        for (int j = 0; j < JN; ++j)
          st.w[j] = lora_ranks(lb, ((size_t)a * P.n + min(n0 + wn + 32 * j + lr, P.n - 1)) * P.r, (size_t)P.adapters * P.n * P.r, p0, P.r);
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
          for (int e = 0; e < EPC / 4; ++e) {              // (a row of another adapter: zeros; rp is a multiple of two chunks)
            st.t[i][e] = u32x4_t{0, 0, 0, 0};
            if (rows >> (32 * i + lr) & 1) st.t[i][e] = *reinterpret_cast<const u32x4_t*>(P.T + (size_t)(m0 + wm + 64 * h + 32 * i + lr) * P.rp + p0 + 4 * e);
          }
        p += 2 * EPC;
        return true;
      };
      auto multiply = [&](const Step& st) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < H; ++i) {
          u32x4_t part[3];                                 // (cut off, not rounded: 3 x 8 bits are all 24, and the largest values stay finite; an infinity is its first part)
          if constexpr (sizeof(E) == 2) {
            float x[EPC];
#pragma unroll
            for (int e = 0; e < EPC; ++e) x[e] = __uint_as_float(st.t[i][e / 4][e % 4]);
#pragma unroll
            for (int q = 0; q < 3; ++q)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float y = __uint_as_float(__float_as_uint(x[2 * e]) & 0xffff0000u), z = __uint_as_float(__float_as_uint(x[2 * e + 1]) & 0xffff0000u);
                part[q][e] = __float_as_uint(y) >> 16 | __float_as_uint(z);
                x[2 * e] = x[2 * e] == y ? 0.f : x[2 * e] - y;
                x[2 * e + 1] = x[2 * e + 1] == z ? 0.f : x[2 * e + 1] - z;
              }
          }
          const uint32_t of = (uint32_t)(st.rows >> (32 * i)) >> (4 * lg);
#pragma unroll
          for (int j = 0; j < JN; ++j) {
            floatx16_t d;
#pragma unroll
            for (int r = 0; r < 16; ++r) d[r] = 0.f;
            if constexpr (sizeof(E) == 2) {
#pragma unroll
              for (int q = 2; q >= 0; --q) lora_mma32(E{}, d, part[q], st.w[j]);
            } else {
              lora_mma32(E{}, d, st.t[i][0], st.w[j]);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[H * h + i][j][r] += of >> (8 * (r >> 2) + (r & 3)) & 1 ? d[r] : 0.f;
          }
        }
      };
      Step one, two;
      if constexpr (JN > 2) {                              // (two steps' registers are not there beside 64 x 128 accumulators)
        while (next(one)) multiply(one);
        continue;
      }
      bool more = next(one);
      while (more) {
        more = next(two);
        multiply(one);
        if (!more) break;
        more = next(one);
        multiply(two);
      }
    }
  }

  if (s0 < s1) {
    if (s0 + S - 1 < s1) pg_wait<NL * (S - 1)>(); else pg_wait<0>();
    lds_barrier();
    frags(0, 0, 0);
  }
  int slot = 0;
  for (int s = s0; s < s1; ++s) {
    const int nslot = slot + 1 == S ? 0 : slot + 1;
#pragma unroll
    for (int k = 0; k < NKK; ++k) {
      if (k + 1 < NKK) {
        frags((k + 1) & 1, slot, k + 1);
      } else if (s + 1 < s1) {                 // every fragment of this step is read: its place in the ring is free once all waves say so
        if (s + S - 1 < s1) pg_wait<NL * (S - 2)>(); else pg_wait<0>();
        lds_barrier();
        if (s + S < s1) issue(s + S, slot);
        frags((k + 1) & 1, nslot, 0);
      }
#pragma unroll
      for (int j = 0; j < JN; ++j)
#pragma unroll
        for (int i = 0; i < IM; ++i) lora_mma32(E{}, acc[i][j], fa[k & 1][i], fb[k & 1][j]);
    }
    static_assert(NKK % 2 == 0, "a step ends on the buffer that the next begins with");
    slot = nslot;
  }

  // Through a descriptor that ends with the tile's last row: rows past m (and, by an offset out of its range, columns past n) read as zeros and are not written.
  float* const to = P.ks == 1 ? P.C : P.part + (size_t)slice * P.m * P.n;
  const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(to + (size_t)m0 * P.n, (short)0, rowsA * P.n * 4, 0x00020000);
  const bool add = P.ks == 1 && P.accumulate;
#pragma unroll
  for (int j = 0; j < JN; ++j) {
    const int col = n0 + wn + j * 32 + lr;
    const uint32_t cb = (uint32_t)(wm + 4 * lg) * P.n * 4 + (col < P.n ? col * 4u : 0x40000000u);
#pragma unroll
    for (int i = 0; i < IM; ++i) {
      float old[16];
      auto at = [&](int r) __attribute__((always_inline)) {
        uint32_t x = cb;
        asm volatile("" : "+v"(x));              // (formed where it is used: kept from a load to its store, the offsets take registers)
        return (int)(x + (uint32_t)(i * 32 + 8 * (r >> 2) + (r & 3)) * P.n * 4);
      };
#pragma unroll
      for (int r = 0; r < 16; ++r) old[r] = 0.f;
      if (add)
#pragma unroll
        for (int r = 0; r < 16; ++r) old[r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rc, at(r), 0, 0));
#pragma unroll
      for (int r = 0; r < 16; ++r) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(old[r] + acc[i][j][r]), rc, at(r), 0, 0);
    }
  }
}

}  // namespace first
