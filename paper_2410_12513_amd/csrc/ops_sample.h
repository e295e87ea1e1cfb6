// Draws with temperature, top-k, top-p and min-p (first_sample); the uniform numbers are the caller's.
//
// The tokens of a row stand in order of their logits, largest first, equal ones by index; a token weighs w = exp((l - l_max) / T).
// Each rule keeps a prefix of that order: the first top_k; of those, the tokens before which less than top_p of their mass lies; the
// weights >= min_p.  The shortest prefix is what is drawn from: the first token whose cumulative weight exceeds u times the prefix's.
//
// So everything is one question, asked of counts or of masses: at which token does the running sum pass a target?  Masses are whole
// numbers (a weight is rounded to a multiple of 2^-S, S such that a row's sum fits 62 bits): their sums do not depend on the order of
// additions, and a token's share is off by 2^-S-1 at most, 1e-14 at 128256 tokens.  32-bit sums would put one draw in some 10^4 of a flat
// row of that size beside its token.
//
// 256 rows of 128256 logits, top_p: 97 us, floor 26 (131 MB): a workgroup, so a compute unit, a row.  60 % of the time its vector units issue: some 30 instructions a logit
// for the masses, ten for the list, four for the maximum; the rest is a row's own chain, sort and sums of the list (a fifth), which no other row fills in for.
// One row of 32000 logits with all rules: 13 to 17 us by box, that chain.
#pragma once
#include "common.h"

namespace first {

struct SampleArgs {
  const float* logits;
  long long pitch;
  int vocab, index_bits, S;               // index_bits: of vocab - 1
  int held;                               // pieces of a thread that LDS holds
  const float *uniforms, *temperature;    // per row; temperature, top_k, top_p, min_p may be null
  const int* top_k;
  const float *top_p, *min_p;
  int* token;
  float* logprob;                         // may be null
  int* kept;                              // may be null
};

constexpr int SR_THREADS = 1024, SR_WAVES = SR_THREADS / 64, SR_BINS = 2048;

struct SrSum { unsigned long long mass; unsigned count; };
__device__ __forceinline__ SrSum operator+(SrSum a, SrSum b) { return {a.mass + b.mass, a.count + b.count}; }
__device__ __forceinline__ SrSum sr_shfl_up(SrSum a, int d) { return {(unsigned long long)__shfl_up((long long)a.mass, d, 64), (unsigned)__shfl_up((int)a.count, d, 64)}; }
__device__ __forceinline__ SrSum sr_shfl_xor(SrSum a, int d) { return {(unsigned long long)__shfl_xor((long long)a.mass, d, 64), (unsigned)__shfl_xor((int)a.count, d, 64)}; }

// Ascending with the logit (-0 counts as 0).
__device__ __forceinline__ uint32_t sr_order(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float sr_value(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o); }

struct SrRow {                            // what a row's weights are made of
  float lmax;
  double c;                               // log2 e / T
  int S;
  // log2 of the weight of a logit that is neither NaN nor -inf
  __device__ __forceinline__ double log2w(float l) const { return l == lmax ? 0.0 : ((double)l - (double)lmax) * c; }
  // tokens that count at all: the weight is not 0 in 64 bits (half of the smallest number, 2^-1075, is rounded to 0, more than that is not)
  __device__ __forceinline__ bool counts(float l, double x) const { return l > -INFINITY && x > -1075.0; }
  // 2^t.  f, the rest of t to the nearest whole number: 2^f = 1 + f q(f), q of degree 9 through the Chebyshev points of [-1/2, 1/2] (6e-16)
  // (the numbers opaque in scalar registers: seen as constants they are copied to a vector register before every step, nine more instructions)
  __device__ __forceinline__ static double series(double f) {
    auto k = [](double v) __attribute__((always_inline)) { asm("" : "+s"(v)); return v; };
    double p = k(7.070977963327673e-09);
    p = fma(p, f, k(1.0205905547945269e-07));
    p = fma(p, f, k(1.3215451634133493e-06));
    p = fma(p, f, k(1.5252672924230416e-05));
    p = fma(p, f, k(0.00015403530424769424));
    p = fma(p, f, k(0.001333355820079545));
    p = fma(p, f, k(0.00961812910761868));
    p = fma(p, f, k(0.05550410866465167));
    p = fma(p, f, k(0.24022650695910075));
    p = fma(p, f, k(0.6931471805599462));
    return fma(p, f, 1.0);
  }
  __device__ __forceinline__ static double power(double t) {
    const double n = rint(t);
    return ldexp(series(t - n), (int)n);
  }
  // The weight times 2^S as a whole number; 0 for NaN and -inf.  The largest logit must be finite here, or l is it.
  __device__ __forceinline__ unsigned long long mass(float l) const {
    return whole(fmax(l == INFINITY ? (double)S : fma((double)l - (double)lmax, c, (double)S), -64.0));
  }
  // 2^t as a whole number, t <= 50 not far below 0: f and q as above, and the sum with 2^(52 - n), n the whole part of t, leaves 2^n (1 + f q(f)) rounded in its low bits
  __device__ __forceinline__ static unsigned long long whole(double t) {
    const double x = 6755399441055744.0 - t, f = t + (x - 6755399441055744.0);           // (3 2^51: -n in the low bits of x)
    const double y = series(f) + __hiloint2double((__double2loint(x) << 20) + ((1023 + 52) << 20), 0);
    return (unsigned long long)__double_as_longlong(y) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ bool heavy(double x, float min_p) const { return power(fmax(x, -1100.0)) >= (double)min_p; }
};

struct SrFound { float value; int index; SrSum through; };   // the token at which the sum passes the target, and the sum up to and with it

struct SrShared {
  unsigned long long mass[SR_BINS];
  unsigned count[SR_BINS];
  SrSum wave[SR_WAVES];
  SrSum before;
  int bin;
};

__device__ __forceinline__ SrSum sr_block_sum(SrSum v, SrShared& sh) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = v + sr_shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.wave[threadIdx.x >> 6] = v;
  __syncthreads();
  SrSum t = {0, 0};
  for (int w = 0; w < SR_WAVES; ++w) t = t + sh.wave[w];
  return t;
}

// The first token in the order at which the running count (by_mass: the running mass) exceeds target; target is below the row's total.
// Digit by digit of (logit, index): a histogram of the tokens that share the digits found so far, and the bin that the sum passes the target in.
__device__ inline SrFound sr_find(const float* row, int V, int index_bits, const SrRow& R, bool by_mass, unsigned long long target, SrShared& sh) {
  const int tid = threadIdx.x;
  uint32_t hi = 0, hi_mask = 0, at = 0, at_mask = 0;
  SrSum before = {0, 0};
  const int index_levels = (index_bits + 10) / 11;
  for (int level = 0; level < 3 + index_levels; ++level) {
    const bool on_logit = level < 3;
    const int shift = on_logit ? (level == 0 ? 21 : level == 1 ? 10 : 0) : 11 * (2 + index_levels - level);
    const uint32_t digit = on_logit && level == 2 ? 0x3ffu : 0x7ffu;
    __syncthreads();
    for (int i = tid; i < SR_BINS; i += SR_THREADS) { sh.mass[i] = 0ull; sh.count[i] = 0u; }
    __syncthreads();
    for (int i = tid; i < V; i += SR_THREADS) {
      const float l = row[i];
      const uint32_t o = sr_order(l);
      if (!(l > -INFINITY) || (o & hi_mask) != hi || ((uint32_t)i & at_mask) != at) continue;
      const double x = R.log2w(l);
      if (!R.counts(l, x)) continue;
      const int bin = on_logit ? (int)(digit - (o >> shift & digit)) : (int)((uint32_t)i >> shift & digit);
      atomicAdd(&sh.count[bin], 1u);
      atomicAdd(&sh.mass[bin], R.mass(l));
    }
    __syncthreads();
    // two bins a thread: the running sum, and the one that passes
    const SrSum a = {sh.mass[2 * tid], sh.count[2 * tid]}, b = {sh.mass[2 * tid + 1], sh.count[2 * tid + 1]};
    SrSum incl = a + b;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const SrSum o = sr_shfl_up(incl, d);
      if ((tid & 63) >= d) incl = incl + o;
    }
    if ((tid & 63) == 63) sh.wave[tid >> 6] = incl;
    __syncthreads();
    SrSum base = before;
    for (int w = 0; w < tid >> 6; ++w) base = base + sh.wave[w];
    incl = base + incl;
    const SrSum s1 = incl, s0 = {s1.mass - b.mass, s1.count - b.count}, sb = {s0.mass - a.mass, s0.count - a.count};
    auto past = [&](SrSum s) { return (by_mass ? s.mass : (unsigned long long)s.count) > target; };
    if (past(s0) && !past(sb)) { sh.bin = 2 * tid; sh.before = sb; }
    if (past(s1) && !past(s0)) { sh.bin = 2 * tid + 1; sh.before = s0; }
    __syncthreads();
    before = sh.before;
    const uint32_t bin = (uint32_t)sh.bin;
    if (on_logit) { hi |= (digit - bin) << shift; hi_mask |= digit << shift; }
    else { at |= bin << shift; at_mask |= digit << shift; }
  }
  const float value = sr_value(hi);
  return {value, (int)at, before + SrSum{R.mass(value), 1u}};
}

// ---- a row in three looks --------------------------------------------------------------------------------------------------
// What can be drawn and where the cuts lie is decided among a few tokens, a list in LDS that is put in order; what is not on it only matters by its sum.
//   with top_k (up to SR_TOPK): the k-th largest of the maxima of threads, or of groups of 2 to 16 of them, is a bound that at least k tokens reach; the
//     list is what reaches it, and no other weight is formed;
//   else: a histogram of the masses over 4096 equal parts of the range of logits that weigh anything says in which part each cut lies, and in which few the draw
//     can lie; the list is those parts' tokens.
// A list that does not fit (masses of equal logits, logits that crowd one part) is left for the digit by digit search over the whole row.
constexpr int SR_LIST = 4096, SR_TOPK = 960, SR_U = 4, SR_PARTS = 4096;
struct __align__(4) SrFour { float v[4]; };               // (a row starts on 4 bytes)

struct SrFast {
  union { unsigned long long list[SR_LIST], hist[SR_PARTS]; };            // (the histogram is through before the list begins)
  unsigned long long wave[SR_WAVES], base_c, base_d, total, kept_mass;
  int found, first_c, cut_p, cut_m, kept, pick, c1, c2, d1, d2;
  unsigned count[SR_WAVES];
  float lo[SR_WAVES], hi[SR_WAVES];
};
union SrLds { SrShared slow; SrFast fast; };

// The row in pieces of four logits, a thread's own ones 4 * SR_THREADS logits apart: four(piece, index of its first logit) of each, and one(logit, index) of what
// fills no piece; SR_U pieces are looked at while the next SR_U are on their way.  FIRST: the thread's first `held` pieces go to LDS, where later looks find them.
constexpr int SR_HELD = 7;
struct SrHeld { float4* lds; int n; };
template <bool FIRST, typename F, typename G> __device__ __forceinline__ void sr_each(const float* row, int V, SrHeld held, F four, G one) {
  const int pieces = V / 4, tid = threadIdx.x, mine = pieces > tid ? (pieces - tid + SR_THREADS - 1) / SR_THREADS : 0;
  SrFour a[SR_U], b[SR_U];
  auto fetch = [&](SrFour (&x)[SR_U], int i) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < SR_U; ++u) x[u] = *reinterpret_cast<const SrFour*>(row + 4 * (tid + SR_THREADS * min(i + u, mine - 1)));     // (past the end: a piece there is)
  };
  auto look = [&](const SrFour (&x)[SR_U], int i) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < SR_U; ++u)
      if (i + u < mine) {
        if (FIRST && i + u < held.n) held.lds[(i + u) * SR_THREADS + tid] = make_float4(x[u].v[0], x[u].v[1], x[u].v[2], x[u].v[3]);
        four(x[u], 4 * (tid + SR_THREADS * (i + u)));
      }
  };
  const float last = tid < V - 4 * pieces ? row[4 * pieces + tid] : 0.f;
  const int i0 = FIRST ? 0 : held.n;
  if (i0 < mine) fetch(a, i0);
  if (!FIRST)
    for (int u = 0; u < min(held.n, mine); ++u) {
      const float4 x = held.lds[u * SR_THREADS + tid];
      four(SrFour{{x.x, x.y, x.z, x.w}}, 4 * (tid + SR_THREADS * u));
    }
  for (int i = i0; i < mine; i += 2 * SR_U) {
    if (i + SR_U < mine) fetch(b, i + SR_U);
    look(a, i);
    if (i + 2 * SR_U < mine) fetch(a, i + 2 * SR_U);
    if (i + SR_U < mine) look(b, i + SR_U);
  }
  if (tid < V - 4 * pieces) one(last, 4 * pieces + tid);
}
template <typename F> __device__ __forceinline__ void sr_each(const float* row, int V, SrHeld held, F f) {
  sr_each<false>(row, V, held, [&](const SrFour& x, int i) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f(x.v[e], i + e);
  }, f);
}
__device__ __forceinline__ unsigned long long sr_key(float l, int i) { return (unsigned long long)sr_order(l) << 32 | (uint32_t)~i; }

// list[0 .. n) into descending order, n <= SR_LIST.  Ends with a barrier.
__device__ inline void sr_sort(unsigned long long* list, int n) {
  const int tid = threadIdx.x;
  if (n <= 128) {                                          // by rank: a key's place is the number of larger ones (all differ but for zeros)
    const unsigned long long x = tid < n ? list[tid] : 0ull;
    int before = 0;
    if (tid < n)
      for (int j = 0; j < n; ++j) before += list[j] > x;
    __syncthreads();
    if (tid < n) list[tid] = 0ull;                         // (places behind equal zeros)
    __syncthreads();
    if (tid < n) list[before] = x;
    __syncthreads();
    return;
  }
  int size = 256;
  while (size < n) size *= 2;
  for (int i = n + tid; i < size; i += SR_THREADS) list[i] = 0ull;
  __syncthreads();
  for (int k = 1; 1 << k <= size; ++k)
    for (int j = k - 1; j >= 0; --j) {
      for (int t = tid; t < size / 2; t += SR_THREADS) {
        const int i = (t >> j << (j + 1)) + (t & ((1 << j) - 1)), o = i + (1 << j);
        const unsigned long long a = list[i], b = list[o];
        if ((a < b) == ((i >> k & 1) == 0)) { list[i] = b; list[o] = a; }
      }
      // (pairs up to 64 apart: a wave's own 128 keys)
      if (j >= 7 || j == 0) __syncthreads();
      else { __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront"); __builtin_amdgcn_wave_barrier(); }
    }
}
// Running sum over the lanes of a wave, in the lanes themselves (rows of 16, then their last lanes handed on).
__device__ __forceinline__ unsigned long long sr_wave_sums(unsigned long long v) {
#define FIRST_SUM_STEP(CTRL, ROWS)                                                                                 \
  {                                                                                                                \
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);         \
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false); \
    v += ((unsigned long long)hi << 32) | lo;                                                                      \
  }
  FIRST_SUM_STEP(0x111, 0xf) FIRST_SUM_STEP(0x112, 0xf) FIRST_SUM_STEP(0x114, 0xf) FIRST_SUM_STEP(0x118, 0xf)
  FIRST_SUM_STEP(0x142, 0xa) FIRST_SUM_STEP(0x143, 0xc)
#undef FIRST_SUM_STEP
  return v;
}
// Exclusive running sum over the threads, and the sum of all.
__device__ __forceinline__ unsigned long long sr_scan(unsigned long long v, unsigned long long* wave, unsigned long long& all) {
  const int tid = threadIdx.x, lane = tid & 63;
  const unsigned long long incl = sr_wave_sums(v);
  __syncthreads();
  if (lane == 63) wave[tid >> 6] = incl;
  __syncthreads();
  static_assert(SR_WAVES == 16, "a row of lanes holds the waves' sums");
  const unsigned long long w = sr_wave_sums(lane < SR_WAVES ? wave[lane] : 0ull);
  const int before = __builtin_amdgcn_readfirstlane((tid >> 6) - 1);
  auto at = [&](int l) { return ((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(w >> 32), l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)w, l); };
  all = at(SR_WAVES - 1);
  return (before >= 0 ? at(max(before, 0)) : 0ull) + incl - v;
}
// Whole numbers of a fraction of a mass: what a running sum has to reach (at least 1), and what it has to pass.
__device__ __forceinline__ unsigned long long sr_reach(float p, unsigned long long total) {
  const double want = ceil(fmax((double)p, 0.0) * (double)total);
  const unsigned long long x = want < 1.0 ? 1ull : (unsigned long long)want;
  return x < total ? x : total;
}
__device__ __forceinline__ unsigned long long sr_pass(float u, unsigned long long total) {
  const double want = floor(fmax((double)u, 0.0) * (double)total);
  const unsigned long long x = want < (double)total ? (unsigned long long)want : total;
  return x < total ? x : total - 1;
}

struct SrRules { float u, top_p, min_p; int top_k; bool greedy; };
struct SrOut { int token; float value; unsigned long long kept_mass; int kept; };

// Equal parts of [lmax - range, lmax], a logit's part is (lmax - l) times this; what weighs less than 2^-66 is in the last one.
__device__ __forceinline__ float sr_parts(const SrRow& R, float lmin) {
  const float all = (float)(66.0 / R.c), range = R.lmax - lmin > 1e-30f ? fminf(R.lmax - lmin, all) : all;
  return range > 1e-30f && range < INFINITY ? (SR_PARTS - 1) / range : 0.f;
}
struct SrFirst { float value; int index; };                // a thread's own largest logit, and an index that is its or a little larger
// False: the list did not fit.
__device__ __forceinline__ bool sr_fast(const float* row, int V, SrHeld held, const SrRow& R, const SrRules& Q, SrFirst first, float lmin, SrFast& sh, SrOut& out) {
  const int tid = threadIdx.x;
  const bool by_prefix = Q.top_k > 0 && Q.top_k <= SR_TOPK, whole = V <= 512 || (V <= SR_LIST && Q.top_k > SR_TOPK);      // (512: put in order in one go)
  const bool cut_p = !Q.greedy && Q.top_p < 1.f, cut_m = !Q.greedy && Q.min_p > 0.f;
  if (Q.top_k > SR_TOPK && Q.top_k < V && !whole) return false;
  if (!(whole || by_prefix) && !(R.lmax < INFINITY)) return false;
  if (tid == 0) { sh.found = 0; sh.first_c = 0; sh.base_c = sh.base_d = 0ull; sh.c1 = 0; sh.c2 = SR_PARTS; sh.d1 = 0; sh.d2 = SR_PARTS; }
  __syncthreads();
  if (whole || by_prefix) {
    unsigned long long bound = 0ull;
    if (!whole) {
      unsigned long long own = first.value > -INFINITY ? sr_key(first.value, first.index) : 0ull;
      // groups of g threads: as large as leaves some more groups with tokens than the bound has to count
      int g = 16;
      while (g > 1 && (SR_THREADS / g < Q.top_k + Q.top_k / 4 || V / (4 * g) < Q.top_k + Q.top_k / 4)) g /= 2;
      for (int d = 1; d < g; d *= 2) {
        const unsigned long long o = (unsigned long long)__shfl_xor((long long)own, d, 64);
        own = o > own ? o : own;
      }
      if (tid % g == 0) sh.list[tid / g] = own;
      __syncthreads();
      sr_sort(sh.list, SR_THREADS / g);                    // (the zeros of threads without a token stand behind the others)
      bound = sh.list[Q.top_k - 1];
      __syncthreads();
    }
    if (whole) {                                           // (what is no token: 0, behind the others)
      for (int i = tid; i < V; i += SR_THREADS) sh.list[i] = row[i] > -INFINITY ? sr_key(row[i], i) : 0ull;
      if (tid == 0) sh.found = V;
    } else {
      const float least = bound != 0 ? sr_value((uint32_t)(bound >> 32)) : -3.402823466e38f;
      sr_each(row, V, held, [&](float l, int i) {
        if (!(l >= least)) return;                         // (nor NaN and -inf)
        const unsigned long long key = sr_key(l, i);
        if (key < bound) return;
        const int to = atomicAdd(&sh.found, 1);
        if (to < SR_LIST) sh.list[to] = key;
      });
    }
  } else {
    // masses over equal parts of [lmax - range, lmax]; what weighs less than 2^-66 is in the last part
    const float inv = sr_parts(R, lmin);
    auto part = [&](float l) __attribute__((always_inline)) { return (int)fminf((R.lmax - l) * inv, (float)(SR_PARTS - 1)); };
    for (int i = tid; i < SR_PARTS; i += SR_THREADS) sh.hist[i] = 0ull;
    __syncthreads();
    // (what weighs nothing would crowd the last part: zeros are spread over the threads' own)
    const float lowest = fmaxf((float)((double)R.lmax - (R.S + 2) / R.c * (1.0 + 1e-6)), -3.402823466e38f);
    const double c = R.c, top = R.lmax, S = R.S;
    auto mass = [&](float l) __attribute__((always_inline)) { return SrRow::whole(fmax(fma((double)l - top, c, S), -64.0)); };
    auto bin = [&](float l) __attribute__((always_inline)) { return l >= lowest ? part(l) : tid; };
    sr_each<false>(row, V, held, [&](const SrFour& x, int) {
      unsigned long long w[4];
      int to[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) { w[e] = mass(x.v[e]); to[e] = bin(x.v[e]); }
#pragma unroll
      for (int e = 0; e < 4; ++e) atomicAdd(&sh.hist[to[e]], w[e]);
    }, [&](float l, int) { atomicAdd(&sh.hist[bin(l)], mass(l)); });
    __syncthreads();
    unsigned long long h[4], total;                        // four parts a thread: the sums through them
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = sh.hist[4 * tid + e] + (e > 0 ? h[e - 1] : 0ull);
    const unsigned long long before = sr_scan(h[3], sh.wave, total);
    auto sum_before = [&](int e) __attribute__((always_inline)) { return before + (e > 0 ? h[e - 1] : 0ull); };
    if (cut_m) {                                           // the parts in which w = min_p can lie
      const double l = (double)R.lmax + log2((double)Q.min_p) / R.c, off = 1e-6 * (fabs(l) + fabs((double)R.lmax));
      const int a = part((float)(l + off)), b = part((float)(l - off));
      if (tid == 0) { sh.c1 = min(a, b); sh.c2 = max(a, b); }
    }
    // the first part at which the sum reaches x: f(part, sum before it)
    auto at = [&](unsigned long long x, auto f) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (sum_before(e) < x && x <= before + h[e]) f(4 * tid + e, sum_before(e));
    };
    __syncthreads();
    if (cut_p) {
      const int c1 = sh.c1, c2 = sh.c2;
      __syncthreads();
      at(sr_reach(Q.top_p, total), [&](int i, unsigned long long) {
        if (!cut_m || i < c1) { sh.c1 = i; sh.c2 = i; }
        else if (i <= c2) sh.c2 = c2;
      });
      __syncthreads();
    }
    const bool cut = cut_p || cut_m;
    // sums before c1 and through c2: what is kept lies between
    if (cut) {
      const int c1 = sh.c1, c2 = sh.c2;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (4 * tid + e == c1) sh.base_c = sum_before(e);
        if (4 * tid + e == c2) sh.total = before + h[e];
      }
    } else if (tid == 0) {
      sh.base_c = sh.total = total;
      sh.c1 = sh.c2 = SR_PARTS;
    }
    __syncthreads();
    const unsigned long long least = sh.base_c, largest = sh.total;
    at(least > 0 ? sr_pass(Q.u, least) + 1 : 1ull, [&](int i, unsigned long long b) { sh.d1 = i; sh.base_d = b; });
    at(sr_pass(Q.u, largest) + 1, [&](int i, unsigned long long) { sh.d2 = i; });
    __syncthreads();
    const int c1 = sh.c1, c2 = sh.c2, d1 = sh.d1, d2 = sh.d2;
    unsigned ahead = 0;                                    // tokens before c1; without cuts, all
    // (a part is where min((lmax - l) inv, last) ends up when cut off: in whole steps of the bounds)
    const float fc1 = (float)c1, fc2 = (float)(c2 + 1), fd1 = (float)d1, fd2 = (float)(d2 + 1);
    auto wanted = [&](float l) __attribute__((always_inline)) {
      const float y = fminf((R.lmax - l) * inv, (float)(SR_PARTS - 1));
      ahead += cut ? y < fc1 : R.counts(l, R.log2w(l));
      return ((int)(y >= fc1) & (int)(y < fc2)) | ((int)(y >= fd1) & (int)(y < fd2));
    };
    auto take = [&](float l, int i) __attribute__((always_inline)) {
      if (!(l > -INFINITY)) return;
      const int to = atomicAdd(&sh.found, 1);
      if (to < SR_LIST) sh.list[to] = sr_key(l, i);
    };
    sr_each<false>(row, V, held, [&](const SrFour& x, int i) {
      int is[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) is[e] = wanted(x.v[e]);
      if (is[0] | is[1] | is[2] | is[3])
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (is[e]) take(x.v[e], i + e);
    }, [&](float l, int i) {
      if (wanted(l)) take(l, i);
    });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) ahead += (unsigned)__shfl_xor((int)ahead, d, 64);
    if ((tid & 63) == 0) sh.count[tid >> 6] = ahead;
    if (tid == 0) sh.total = total;
  }
  __syncthreads();
  const int n = sh.found;
  if (n > SR_LIST) return false;
  sr_sort(sh.list, n);

  // The list in order, four tokens a thread: running sums.  by parts: the draw's tokens come first, then (or among them) the cuts'; sums start at the parts' own.
  const bool lists_all = whole || by_prefix;
  const float inv = sr_parts(R, lmin);
  const int c1 = sh.c1, d2 = sh.d2;
  const bool apart = !lists_all && d2 + 1 < c1;            // the cuts' parts do not touch the draw's
  const int limit = Q.top_k > 0 ? Q.top_k : SR_LIST;
  float value[4];
  unsigned long long w[4], sum = 0, in_d = 0;
  int cnt = 0, in_c = 0;
  bool ok[4], c_part[4], heavy[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = 4 * tid + e;
    const unsigned long long key = i < n ? sh.list[i] : 0ull;
    value[e] = sr_value((uint32_t)(key >> 32));
    const double x = R.log2w(value[e]);
    ok[e] = i < n && (!lists_all || i < limit) && R.counts(value[e], x);
    w[e] = ok[e] ? R.mass(value[e]) : 0ull;
    heavy[e] = ok[e] && (!cut_m || R.heavy(x, Q.min_p));
    const int b = lists_all ? 0 : (int)fminf((R.lmax - value[e]) * inv, (float)(SR_PARTS - 1));
    c_part[e] = lists_all || b >= c1;
    sum += w[e];
    in_d += c_part[e] ? 0ull : w[e];
    cnt += ok[e];
    in_c += ok[e] && c_part[e] && heavy[e];
  }
  unsigned long long all, all_d = 0;
  unsigned long long run = sr_scan(sum, sh.wave, all);
  if (!lists_all) sr_scan(in_d, sh.wave, all_d);
  const unsigned long long base = lists_all ? 0ull : sh.base_d, jump = apart ? sh.base_c - (sh.base_d + all_d) : 0ull;      // (what lies between the two)
  const unsigned long long total = lists_all ? all : sh.total;
  run += base;
  unsigned long long cum[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    run += w[e];
    cum[e] = run + (c_part[e] ? jump : 0ull);
  }
  // tokens kept: those ahead of the list, and of the list the first (entries of the cuts' parts)
  unsigned ahead = 0;
  if (!lists_all)
    for (int v = 0; v < SR_WAVES; ++v) ahead += sh.count[v];
  if (tid == 0) { sh.cut_p = 1 << 30; sh.cut_m = 0; sh.first_c = 1 << 30; sh.kept = 0; sh.pick = -1; }
  __syncthreads();
  {
    int first = 1 << 30, counted = 0;
#pragma unroll
    for (int e = 3; e >= 0; --e)
      if (ok[e] && c_part[e]) first = 4 * tid + e;
#pragma unroll
    for (int e = 0; e < 4; ++e) counted += ok[e];
    if (first < 1 << 30) atomicMin(&sh.first_c, first);
    if (in_c) atomicAdd(&sh.cut_m, in_c);
    if (counted) atomicAdd(&sh.kept, counted);
    if (cut_p) {
      const unsigned long long x = sr_reach(Q.top_p, total);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ok[e] && c_part[e] && cum[e] >= x && cum[e] - w[e] < x) atomicMin(&sh.cut_p, 4 * tid + e);
    }
  }
  __syncthreads();
  const bool cut = lists_all || cut_p || cut_m;
  const int first_c = sh.first_c == 1 << 30 ? 0 : sh.first_c, counted = sh.kept;
  int last = lists_all ? counted - 1 : cut ? first_c + sh.cut_m - 1 : -1;                     // the last kept entry
  if (lists_all && cut_m) last = min(last, sh.cut_m - 1);
  if (cut_p) last = min(last, sh.cut_p);
  if (tid == 0 && last < first_c) sh.kept_mass = lists_all ? 0ull : sh.base_c;                // (none of the list)
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (4 * tid + e == last && last >= first_c) sh.kept_mass = cum[e];
  __syncthreads();
  const unsigned long long kept_mass = !cut ? total : sh.kept_mass, target = sr_pass(Q.u, kept_mass);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (ok[e] && cum[e] > target && cum[e] - w[e] <= target && w[e] > 0) {                     // (one token: sums grow)
      sh.pick = 4 * tid + e;
    }
  __syncthreads();
  const int pick = sh.pick;
  if (pick < 0) return false;                              // (cannot be)
  const unsigned long long key = sh.list[pick];
  out.token = (int)~(uint32_t)key;
  out.value = sr_value((uint32_t)(key >> 32));
  out.kept_mass = kept_mass;
  out.kept = !cut ? (int)ahead : (int)ahead + max(0, last - first_c + 1);
  return true;
}

// grid (rows), a workgroup a row.
__global__ void __launch_bounds__(SR_THREADS) k_sample_row(SampleArgs P) {
  __shared__ SrLds lds;
  extern __shared__ __align__(16) char sr_smem[];
  const SrHeld held = {reinterpret_cast<float4*>(sr_smem), P.held};
  const int tid = threadIdx.x, seq = blockIdx.x, V = P.vocab;
  const float* row = P.logits + (size_t)seq * P.pitch;
  SrFirst first = {-INFINITY, 0};
  float lmin = INFINITY;
  // (the index: the last of its piece, which is enough for a bound; the least logit: of every fourth, what lies below it shares the last part)
  sr_each<true>(row, V, held, [&](const SrFour& x, int i) {
    const float top = fmaxf(fmaxf(x.v[0], x.v[1]), fmaxf(x.v[2], x.v[3]));                 // (not NaN where one is a number)
    if (top > first.value) first = {top, i + 3};
    lmin = fminf(lmin, x.v[0] > -INFINITY ? x.v[0] : INFINITY);
  }, [&](float l, int i) {
    if (l > first.value) first = {l, i};
    lmin = fminf(lmin, l > -INFINITY ? l : INFINITY);
  });
  float m = wave_max(first.value);
  lmin = -wave_max(-lmin);
  if ((tid & 63) == 0) { lds.fast.hi[tid >> 6] = m; lds.fast.lo[tid >> 6] = lmin; }
  __syncthreads();
  for (int w = 0; w < SR_WAVES; ++w) { m = fmaxf(m, lds.fast.hi[w]); lmin = fminf(lmin, lds.fast.lo[w]); }
  if (!(m > -INFINITY)) {                 // nothing to draw from
    if (tid == 0) {
      P.token[seq] = -1;
      if (P.logprob) P.logprob[seq] = -INFINITY;
      if (P.kept) P.kept[seq] = 0;
    }
    return;
  }
  const float T = P.temperature ? P.temperature[seq] : 1.f;
  const bool greedy = !(T > 0.f);
  const SrRow R = {m, 1.4426950408889634 / (greedy ? 1.0 : (double)T), P.S};
  SrRules Q = {P.uniforms[seq], P.top_p ? P.top_p[seq] : 1.f, P.min_p ? P.min_p[seq] : 0.f, P.top_k ? max(P.top_k[seq], 0) : 0, greedy};
  if (greedy || Q.min_p > 1.f || Q.top_p <= 0.f) {                       // the first token
    Q.top_k = 1;
    Q.min_p = 0.f;
    Q.top_p = 1.f;
  }
  SrOut out;
  if (!sr_fast(row, V, held, R, Q, first, lmin, lds.fast, out)) {
    __syncthreads();
    SrSum all = {0, 0}, heavy = {0, 0};
    for (int i = tid; i < V; i += SR_THREADS) {
      const float l = row[i];
      const double x = R.log2w(l);
      if (!R.counts(l, x)) continue;
      const SrSum one = {R.mass(l), 1u};
      all = all + one;
      if (R.heavy(x, Q.min_p)) heavy = heavy + one;
    }
    SrShared& sh = lds.slow;
    all = sr_block_sum(all, sh);
    SrSum kept = all;
    if (Q.top_k > 0 && (unsigned)Q.top_k < all.count) kept = sr_find(row, V, P.index_bits, R, false, (unsigned long long)Q.top_k - 1, sh).through;
    if (!greedy && Q.top_p < 1.f) {
      const SrSum p = sr_find(row, V, P.index_bits, R, true, sr_reach(Q.top_p, kept.mass) - 1, sh).through;
      if (p.count < kept.count) kept = p;
    }
    if (!greedy && Q.min_p > 0.f) {
      heavy = sr_block_sum(heavy, sh);
      if (heavy.count < kept.count) kept = heavy;
    }
    const SrFound f = sr_find(row, V, P.index_bits, R, true, sr_pass(Q.u, kept.mass), sh);
    out = {f.index, f.value, kept.mass, (int)kept.count};
  }
  if (tid == 0) {
    P.token[seq] = out.token;
    if (P.logprob) P.logprob[seq] = (float)(R.log2w(out.value) * 0.6931471805599453 - log(ldexp((double)out.kept_mass, -P.S)));
    if (P.kept) P.kept[seq] = out.kept;
  }
}

}  // namespace first
