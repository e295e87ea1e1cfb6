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
#pragma once
#include "common.h"

namespace first {

struct SampleArgs {
  const float* logits;
  long long pitch;
  int vocab, index_bits, S;               // index_bits: of vocab - 1
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
  // tokens that count at all: the weight is not 0 in 64 bits
  __device__ __forceinline__ bool counts(float l, double x) const { return l > -INFINITY && x > -1074.5; }
  __device__ __forceinline__ unsigned long long mass(double x) const { return (unsigned long long)rint(ldexp(exp2(x), S)); }
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
      atomicAdd(&sh.mass[bin], R.mass(x));
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
  return {value, (int)at, before + SrSum{R.mass(R.log2w(value)), 1u}};
}

// grid (rows), a workgroup a row.
__global__ void __launch_bounds__(SR_THREADS) k_sample_row(SampleArgs P) {
  __shared__ SrShared sh;
  __shared__ float wmax[SR_WAVES];
  const int tid = threadIdx.x, seq = blockIdx.x, V = P.vocab;
  const float* row = P.logits + (size_t)seq * P.pitch;
  float m = -INFINITY;
  for (int i = tid; i < V; i += SR_THREADS) m = fmaxf(m, row[i]);          // (fmaxf passes over NaN)
  m = wave_max(m);
  if ((tid & 63) == 0) wmax[tid >> 6] = m;
  __syncthreads();
  for (int w = 0; w < SR_WAVES; ++w) m = fmaxf(m, wmax[w]);
  if (!(m > -INFINITY)) {                 // nothing to draw from
    if (tid == 0) {
      P.token[seq] = -1;
      if (P.logprob) P.logprob[seq] = -INFINITY;
      if (P.kept) P.kept[seq] = 0;
    }
    return;
  }
  const float T = P.temperature ? P.temperature[seq] : 1.f, u = P.uniforms[seq];
  const bool greedy = !(T > 0.f);
  const SrRow R = {m, greedy ? 0.0 : 1.4426950408889634 / (double)T, P.S};
  const float min_p = P.min_p ? P.min_p[seq] : 0.f, top_p = P.top_p ? P.top_p[seq] : 1.f;
  const int top_k = greedy ? 1 : P.top_k ? P.top_k[seq] : 0;
  SrSum all = {0, 0}, heavy = {0, 0};
  for (int i = tid; i < V; i += SR_THREADS) {
    const float l = row[i];
    if (!(l > -INFINITY)) continue;
    const double x = R.log2w(l);
    if (!R.counts(l, x)) continue;
    const SrSum one = {R.mass(x), 1u};
    all = all + one;
    if (exp2(x) >= (double)min_p) heavy = heavy + one;
  }
  all = sr_block_sum(all, sh);
  SrSum kept = all;
  if (top_k > 0 && (unsigned)top_k < all.count) kept = sr_find(row, V, P.index_bits, R, false, (unsigned long long)top_k - 1, sh).through;
  if (!greedy && top_p < 1.f) {
    const double want = ceil(fmax((double)top_p, 0.0) * (double)kept.mass);
    const unsigned long long x = want < 1.0 ? 1ull : (unsigned long long)want;
    const SrSum p = sr_find(row, V, P.index_bits, R, true, (x < kept.mass ? x : kept.mass) - 1, sh).through;
    if (p.count < kept.count) kept = p;
  }
  if (!greedy && min_p > 0.f) {
    heavy = sr_block_sum(heavy, sh);
    if (heavy.count == 0) heavy = sr_find(row, V, P.index_bits, R, false, 0, sh).through;     // (min_p > 1: the first token)
    if (heavy.count < kept.count) kept = heavy;
  }
  const double want = floor(fmax((double)u, 0.0) * (double)kept.mass);
  const unsigned long long target = want < (double)kept.mass ? (unsigned long long)want : kept.mass - 1;
  const SrFound f = sr_find(row, V, P.index_bits, R, true, target < kept.mass ? target : kept.mass - 1, sh);
  if (tid == 0) {
    P.token[seq] = f.index;
    if (P.logprob) P.logprob[seq] = (float)(R.log2w(f.value) * 0.6931471805599453 - log(ldexp((double)kept.mass, -P.S)));
    if (P.kept) P.kept[seq] = (int)kept.count;
  }
}

}  // namespace first
