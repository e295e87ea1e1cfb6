// C ABI of the operators of a step over drafted tokens (include/first.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "../../include/first.h"
#include "last_error.h"
#include "ops_lora.h"
#include "ops_rope.h"
#include "ops_sample.h"
#include "ops_tree.h"

using namespace first;

namespace {

// (nothing leaves an entry point: text that finds no memory is dropped)
int refuse(int code, const char* text) noexcept {
  try { g_create_error = text; } catch (...) {}
  return code;
}
int launched(const char* name, hipError_t e = hipSuccess) noexcept {
  const hipError_t last = hipGetLastError();
  if (e == hipSuccess) e = last;
  if (e == hipSuccess) return FIRST_OK;
  try { g_create_error = std::string(name) + ": " + hipGetErrorString(e); } catch (...) {}
  return FIRST_ERR_HIP;
}
bool known_type(int dtype) { return dtype == FIRST_DTYPE_FP32 || dtype == FIRST_DTYPE_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }
size_t size_of(int dtype) { return dtype == FIRST_DTYPE_BF16 ? 2 : 4; }
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

constexpr int CUS = 256;                  // compute units of the MI355X

// Launches; a kernel that may use more than 64 KB of LDS is told so first, once a device: `most` bytes of dynamic LDS in any call (0: lds, always the same).
template <auto kernel, typename Args> hipError_t launch(hipStream_t st, dim3 grid, int threads, size_t lds, const Args& P, size_t most = 0) {
  if (most == 0) most = lds;
  if (most > 32 * 1024) {
    static std::atomic<uint64_t> told{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 64 || !(told.load(std::memory_order_relaxed) >> dev & 1)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
      if (e != hipSuccess) return e;
      if (dev < 64) told.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
  }
  hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, st, P);
  return hipGetLastError();
}

// ---- rotary positions ------------------------------------------------------------------------------------------------------
// Four rows a workgroup where one row leaves threads idle and there are rows enough for every compute unit all the same; else one.  bf16, 16384 rows of heads of 128:
// 8 heads 14.6 us by fours against 18.7, 16 heads 21.5 against 26.8, 40 heads 65.0 against 58.2; 2048 rows of 8 heads 7.2 either way.
template <typename T> hipError_t launch_rope(hipStream_t st, const RopeArgs& P) {
  constexpr int EPC = 16 / (int)sizeof(T);
  const bool whole = (P.interleaved ? P.rot : P.rot / 2) % EPC == 0 && P.hd % EPC == 0 && P.x_pitch % EPC == 0 && P.y_pitch % EPC == 0 && aligned(P.x, 16) && aligned(P.y, 16);
  if (!whole) return launch<&k_rope<T>>(st, dim3(P.rows), WG, 0, P);
  const int items = P.rot / 2 / (P.interleaved ? EPC / 2 : EPC) + (P.hd - P.rot) / EPC;                 // threads' worth of a head
  if (P.heads * items <= WG && P.rows >= 4 * CUS)
    return P.interleaved ? launch<&k_rope_chunks<T, true, 4>>(st, dim3((P.rows + 3) / 4), WG, 0, P) : launch<&k_rope_chunks<T, false, 4>>(st, dim3((P.rows + 3) / 4), WG, 0, P);
  return P.interleaved ? launch<&k_rope_chunks<T, true, 1>>(st, dim3(P.rows), WG, 0, P) : launch<&k_rope_chunks<T, false, 1>>(st, dim3(P.rows), WG, 0, P);
}

// ---- projections with an adapter per row -----------------------------------------------------------------------------------
// stream: up to 32 rows, slices of K such that two workgroups a compute unit are busy, of four steps at least; up to 64 where the slices that fit A's place in LDS stay
// few.  us a call in bf16, stream and the best tile: 16 and 32 x 4096 x 4096 16 and 21; 64 x 688 x 256 10.6 and 12.7; 64 x 14336 x 4096 46.6 and 34.5.
// tile: the BM x BN with the least estimated time, rounds of the chip times the tile's products over how well it feeds the matrix cores; slices of K where the tiles
// of one round leave half of the chip idle.  Tiles of 64 / 128 / 256: 33 x 4096 x 4096 20.9 / 21.9 / 29.3, 250 x 4096 x 4096 37.2 / 30.8 / 37.3 (128 without slices 52),
// 250 x 14336 x 4096 75 / 54.6 / 62.3, 1024 x 4096 x 4096 79.7 / 62.6 / 73.1, 1024 x 14336 x 4096 231 / 194 / 137.
struct LoraPlan { int tile, ks; };        // tile 0: stream
LoraPlan lora_plan(int dtype, int m, int n, int k) {
  const int64_t steps = up((int64_t)k * size_of(dtype), 128) / 128;
  const int64_t groups = (n + 63) / 64, least = up(steps * 128 * (m <= 16 ? 16 : m <= 32 ? 32 : 64), LORA_A_BYTES) / LORA_A_BYTES;     // (a slice of A has to fit its place in LDS)
  if (m <= 32 || (m <= LORA_STREAM_ROWS && least <= 4))
    return {0, (int)std::max(least, std::min((2 * CUS + groups / 2) / groups, steps / 4))};
  LoraPlan best = {64, 1};
  double fastest = 1e300;
  for (int t : {256, 128, 64}) {
    const int64_t tiles = (int64_t)((m + t - 1) / t) * ((n + t - 1) / t);
    const int64_t ks = m > 65535 ? 1 : std::max<int64_t>(1, std::min<int64_t>({CUS / tiles, steps / 8, 8}));
    const double feed = t == 256 ? 1.0 : t == 128 ? 0.75 : 0.38, rounds = (double)((tiles * ks + CUS - 1) / CUS);
    const double time = rounds * ((double)t * t / feed * ((steps + ks - 1) / ks) + 8 * t * t) + (ks > 1 ? 2e5 : 0);
    if (time < fastest) { fastest = time; best = {t, (int)ks}; }
  }
  return best;
}
int lora_rp(int r) { return r <= 16 ? 16 : r <= 32 ? 32 : 64; }
int64_t lora_t_bytes(int m, int r) { return up((int64_t)m * lora_rp(r) * 4, 256); }
template <typename E> hipError_t launch_lora(hipStream_t st, LoraArgs& P, const LoraPlan& plan) {
  P.shrink_tiles = (P.m + 15) / 16;
  P.shrink_ways = std::max(1, std::min(16, CUS / P.shrink_tiles));
  const int helpers = P.shrink_tiles * P.shrink_ways;
  P.ks = plan.ks;
  hipError_t e;
  if (plan.tile == 0) {
    const int grid = helpers + (P.n + 63) / 64 * P.ks;
    const size_t lds = LORA_A_BYTES + 4 * 6 * 2048;
    e = P.m <= 16 ? launch<&k_lora_stream<E, 16, 6>>(st, grid, WG, lds, P) : P.m <= 32 ? launch<&k_lora_stream<E, 32, 6>>(st, grid, WG, lds, P) : launch<&k_lora_stream<E, 64, 6>>(st, grid, WG, lds, P);
  } else {
    e = launch<&k_lora_shrink<E>>(st, helpers, LORA_SHRINK_WAVES * 64, (size_t)LORA_SHRINK_WAVES * 16 * P.rp * 4, P, (size_t)LORA_SHRINK_WAVES * 16 * LORA_RMAX * 4);
    if (e != hipSuccess) return e;
    P.gm = (P.m + plan.tile - 1) / plan.tile;
    P.gn = (P.n + plan.tile - 1) / plan.tile;
    const int grid = P.gm * P.gn * P.ks;
    e = plan.tile == 256 ? launch<&k_lora_tile<E, 256, 256, 4, 2, 128, 2>>(st, grid, 512, 2 * 512 * 128, P)
        : plan.tile == 128 ? launch<&k_lora_tile<E, 128, 128, 4, 2, 128, 4>>(st, grid, 512, 4 * 256 * 128, P)
                           : launch<&k_lora_tile<E, 64, 64, 2, 2, 128, 4>>(st, grid, 256, 4 * 128 * 128, P);
  }
  if (e == hipSuccess && (plan.tile == 0 || P.ks > 1)) e = launch<&k_lora_finish<E>>(st, dim3((P.n + WG - 1) / WG, P.m), WG, 0, P);
  return e;
}

// ---- attention of drafted tokens -------------------------------------------------------------------------------------------
// Rows of a workgroup: the smallest block that holds a sequence's nodes times the query heads of a KV head, up to 256, as its keys are then
// read once (rows of up to 244 over 20000 to 32768 positions in blocks of 256 168 us, of 128 176).  Splits: as many as fill the chip's places for workgroups once (by LDS: two a compute unit up to 80 KB, else one), of whole 128 keys (fp32: 64, whose products take the matrix cores four times as long a bit); twice as
// many splits: 43.6 us against 31 for 16 sequences of 300 to 2300 positions.
struct TreePlan { int block, split_keys, splits, row_blocks, places, step; };
TreePlan tree_plan(const first_tree_attn_desc& d, int B, int max_nodes, int max_len) {
  const int64_t rows = (int64_t)max_nodes * (d.n_q_heads / d.n_kv_heads);
  const bool wide = d.dtype == FIRST_DTYPE_BF16;
  TreePlan p;
  p.block = rows <= 32 ? 32 : rows <= 64 ? 64 : !wide || rows <= 128 ? 128 : 256;
  p.row_blocks = (int)((rows + p.block - 1) / p.block);
  const int places = CUS * (wide && (p.block == 64 || p.block == 128 || d.head_dim == 64) ? 2 : 1);
  const int64_t base = std::max<int64_t>(1, (int64_t)B * d.n_kv_heads * p.row_blocks);
  const int64_t want = std::max<int64_t>(1, places / base);
  const int least = wide ? 128 : 64;
  // Sequences may differ in length (2 to 64 of them): where splits of one length would be longer than the least, the kernel decides from the lengths, down to a quarter as
  // long.  us, one length and so: one of 32768 and 15 of 300 149 and 84, 8 of 4000 to 32000 135 and 118, 4 of 32000 211 and 210, 16 of 1300 27.6 and 28.9.
  p.step = least;
  p.places = B > 1 && B <= 64 && want > 1 && max_len > least * want ? places / d.n_kv_heads : 0;
  const int64_t most = p.places > 0 ? 4 * want : want;
  p.split_keys = (int)std::min<int64_t>(TREE_SPLIT_MAX, std::max<int64_t>(least, up((max_len + most - 1) / most, least)));
  p.splits = std::max(1, (max_len + p.split_keys - 1) / p.split_keys);
  if (p.splits == 1) p.places = 0;
  return p;
}
template <typename E, int HD, int QG, int KH, int NS, int S> hipError_t launch_tree_walk(hipStream_t st, const TreeArgs& P, const TreePlan& p) {
  // (all splits of the greatest length have a place)
  const int64_t least = (int64_t)P.B * p.row_blocks * ((P.max_len + TREE_SPLIT_MAX - 1) / TREE_SPLIT_MAX);
  const dim3 grid = p.places > 0 ? dim3(P.Hkv, (unsigned)std::max<int64_t>(p.places, least), 1) : dim3(P.Hkv * p.row_blocks, p.splits, P.B);
  return launch<&k_tree_attn<E, HD, QG, KH, NS, S>>(st, grid, QG * KH * 64, (size_t)S * 2 * KH * NS * 32 * HD * sizeof(E), P);
}
template <typename E, int HD> hipError_t launch_tree(hipStream_t st, const TreeArgs& P, const TreePlan& p) {
  hipError_t e;
  if constexpr (sizeof(E) == 2) {
    e = p.block == 32 ? launch_tree_walk<E, HD, 1, 4, 1, 2>(st, P, p) : p.block == 64 ? launch_tree_walk<E, HD, 2, 2, 1, 2>(st, P, p)
        : p.block == 128 ? launch_tree_walk<E, HD, 4, 1, 2, 2>(st, P, p) : launch_tree_walk<E, HD, 8, 1, 2, 3>(st, P, p);
  } else {
    e = p.block == 32 ? launch_tree_walk<E, HD, 1, 2, 1, 2>(st, P, p) : p.block == 64 ? launch_tree_walk<E, HD, 2, 2, 1, 2>(st, P, p)
                                                                                        : launch_tree_walk<E, HD, 4, 2, 1, 2>(st, P, p);
  }
  if (e == hipSuccess && p.splits > 1) {
    e = launch<&k_tree_join<E, HD>>(st, dim3((P.max_nodes * P.Hq + WAVES - 1) / WAVES, P.B), WG, 0, P);
  }
  return e;
}

}  // namespace

extern "C" {

int first_op_rope(void* hip_stream, const first_rope_desc* d, const void* x, int64_t x_pitch, void* y, int64_t y_pitch,
                  const int32_t* positions, int32_t rows) {
  if (!d) return refuse(FIRST_ERR_ARG, "first_op_rope: null description");
  if (!known_type(d->dtype) || d->n_heads < 1 || d->n_heads > 65536 || d->head_dim < 2 || d->head_dim > 2 * ROPE_MAX_PAIRS || d->rot_dim < 2 || d->rot_dim % 2 ||
      d->rot_dim > d->head_dim)
    return refuse(FIRST_ERR_ARG, "first_op_rope: unknown dtype, heads outside 1..65536, head_dim outside 2..256, or rot_dim odd or outside 2..head_dim");
  if ((d->layout != FIRST_ROPE_HALF && d->layout != FIRST_ROPE_INTERLEAVED) ||
      (d->scaling != FIRST_ROPE_NONE && d->scaling != FIRST_ROPE_LINEAR && d->scaling != FIRST_ROPE_BANDS))
    return refuse(FIRST_ERR_ARG, "first_op_rope: unknown layout or scaling");
  if (!(d->base > 0.f) || !std::isfinite(d->base) || !std::isfinite(d->amplitude) ||
      (d->scaling != FIRST_ROPE_NONE && (!(d->factor > 0.f) || !std::isfinite(d->factor))) ||
      (d->scaling == FIRST_ROPE_BANDS && (!(d->high > d->low) || !std::isfinite(d->low) || !std::isfinite(d->high) || d->original_len < 1)))
    return refuse(FIRST_ERR_ARG, "first_op_rope: base and factor must be positive, low < high, original_len >= 1, all of them finite");
  const int64_t width = (int64_t)d->n_heads * d->head_dim;
  if (rows < 0 || x_pitch < width || y_pitch < width || x_pitch > INT32_MAX || y_pitch > INT32_MAX)
    return refuse(FIRST_ERR_ARG, "first_op_rope: negative rows, or a pitch below n_heads * head_dim or above 2^31 - 1");
  if (rows == 0) return FIRST_OK;
  if (!x || !y || !positions) return refuse(FIRST_ERR_ARG, "first_op_rope: null pointer");
  const size_t z = size_of(d->dtype);
  if (!aligned(x, z) || !aligned(y, z) || !aligned(positions, 4)) return refuse(FIRST_ERR_ARG, "first_op_rope: a pointer is not on its element's size");
  const char *x0 = (const char*)x, *y0 = (const char*)y;
  const int64_t xn = ((rows - 1) * x_pitch + width) * (int64_t)z, yn = ((rows - 1) * y_pitch + width) * (int64_t)z;
  if (x0 < y0 + yn && y0 < x0 + xn && !(x == y && x_pitch == y_pitch)) {
    // heads side by side in one packed buffer share a range and no element
    const int64_t off = ((y0 - x0) % (x_pitch * (int64_t)z) + x_pitch * (int64_t)z) % (x_pitch * (int64_t)z);
    if (x_pitch != y_pitch || off < width * (int64_t)z || x_pitch * (int64_t)z - off < width * (int64_t)z)
      return refuse(FIRST_ERR_ARG, "first_op_rope: x and y overlap without being the same");
  }
  RopeArgs P;
  P.x = x; P.y = y; P.positions = positions; P.x_pitch = x_pitch; P.y_pitch = y_pitch;
  P.rows = rows; P.heads = d->n_heads; P.hd = d->head_dim; P.rot = d->rot_dim; P.interleaved = d->layout == FIRST_ROPE_INTERLEAVED;
  P.amplitude = d->amplitude; P.sign = d->inverse ? -1.f : 1.f;
  const double two_pi = 6.283185307179586476925, step = -2.0 * std::log((double)d->base) / d->rot_dim;
  double ones[8], eights[ROPE_MAX_PAIRS / 8];               // base^(-2 i / rot_dim) as a product of two: 24 exponentials at most
  for (int i = 0; i < 8; ++i) ones[i] = std::exp(step * i);
  for (int i = 0; 8 * i < d->rot_dim / 2; ++i) eights[i] = std::exp(step * 8 * i);
  for (int i = 0; i < d->rot_dim / 2; ++i) {
    const double f = ones[i % 8] * eights[i / 8];
    double g = f;
    if (d->scaling == FIRST_ROPE_LINEAR) g = f / d->factor;
    if (d->scaling == FIRST_ROPE_BANDS) {
      const double keep = std::min(1.0, std::max(0.0, (d->original_len * f / two_pi - d->low) / ((double)d->high - d->low)));
      g = (1.0 - keep) * f / d->factor + keep * f;
    }
    P.turns[i] = g / two_pi;
  }
  const hipStream_t st = stream_of(hip_stream);
  return launched("first_op_rope", d->dtype == FIRST_DTYPE_BF16 ? launch_rope<bf16>(st, P) : launch_rope<float>(st, P));
}

int64_t first_op_gemm_nt_lora_workspace(int32_t dtype, int32_t m, int32_t n, int32_t k, int32_t r) {
  if (!known_type(dtype) || m < 0 || n < 1 || k < 8 || k % 8 || r < 1 || r > LORA_RMAX)
    return refuse(FIRST_ERR_ARG, "first_op_gemm_nt_lora_workspace: unknown dtype, negative m, n < 1, k not a positive multiple of 8, or rank outside 1..64");
  const LoraPlan plan = lora_plan(dtype, m, n, k);
  return m == 0 ? 0 : lora_t_bytes(m, r) + (plan.tile == 0 || plan.ks > 1 ? (int64_t)plan.ks * m * n * 4 : 0);
}

int first_op_gemm_nt_lora(void* hip_stream, int32_t dtype, const void* A, const void* W, const void* La, const void* Lb, const int32_t* adapter,
                          const float* scale, float* C, int32_t m, int32_t n, int32_t k, int32_t n_adapters, int32_t r, int32_t accumulate, void* workspace,
                          int64_t workspace_bytes) {
  const int64_t need = first_op_gemm_nt_lora_workspace(dtype, m, n, k, r);
  if (need < 0 || n_adapters < 1)
    return refuse(FIRST_ERR_ARG, "first_op_gemm_nt_lora: unknown dtype, negative m, n < 1, k not a positive multiple of 8, rank outside 1..64, or no adapters");
  if (m == 0) return FIRST_OK;
  if (!A || !W || !La || !Lb || !adapter || !scale || !C || !workspace) return refuse(FIRST_ERR_ARG, "first_op_gemm_nt_lora: null pointer");
  if (!aligned(A, 16) || !aligned(W, 16) || !aligned(La, 16) || !aligned(Lb, 16) || !aligned(workspace, 16) || !aligned(C, 4) || !aligned(adapter, 4) || !aligned(scale, 4))
    return refuse(FIRST_ERR_ARG, "first_op_gemm_nt_lora: A, W, La, Lb and the workspace must be on 16 bytes, the others on 4");
  if (workspace_bytes < need) return refuse(FIRST_ERR_CAPACITY, "first_op_gemm_nt_lora: the workspace is smaller than first_op_gemm_nt_lora_workspace says");
  if (m > 1 << 20 || n > 1 << 20 || k > 1 << 20) return refuse(FIRST_ERR_CAPACITY, "first_op_gemm_nt_lora: more than 2^20 rows or columns");
  LoraArgs P = {A, W, La, Lb, adapter, scale, C, (float*)workspace, (float*)((char*)workspace + lora_t_bytes(m, r)), m, n, k, r, lora_rp(r), n_adapters, accumulate != 0};
  const LoraPlan plan = lora_plan(dtype, m, n, k);
  const hipStream_t st = stream_of(hip_stream);
  return launched("first_op_gemm_nt_lora", dtype == FIRST_DTYPE_BF16 ? launch_lora<bf16>(st, P, plan) : launch_lora<float>(st, P, plan));
}

static int tree_refusal(const first_tree_attn_desc* d, int32_t B, int32_t N, int32_t max_nodes, int32_t max_len) {
  if (!d) return refuse(FIRST_ERR_ARG, "first_op_tree_attn: null description");
  if (!known_type(d->dtype) || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads % d->n_kv_heads || d->n_q_heads > 1024 || (d->head_dim != 64 && d->head_dim != 128) ||
      d->page_tokens != TREE_PAGE)
    return refuse(FIRST_ERR_ARG, "first_op_tree_attn: unknown dtype, heads outside 1..1024 or not a multiple of the KV heads, head_dim not 64 or 128, or pages not of 16 tokens");
  if (!std::isfinite(d->scale) || d->n_pages < 0 || d->max_pages < 0 || d->mask_words < 0)
    return refuse(FIRST_ERR_ARG, "first_op_tree_attn: scale not finite, or a negative size");
  if (B < 0 || N < 0 || max_nodes < 0 || max_len < 0) return refuse(FIRST_ERR_ARG, "first_op_tree_attn: a negative size");
  if (B > 65535 || N > 1 << 27) return refuse(FIRST_ERR_CAPACITY, "first_op_tree_attn: more than 65535 sequences or 2^27 nodes");
  if (max_nodes > TREE_MAX_NODES || max_len > 1 << 28) return refuse(FIRST_ERR_CAPACITY, "first_op_tree_attn: more than 2048 nodes of a sequence, or 2^28 positions");
  return FIRST_OK;
}

int64_t first_op_tree_attn_workspace(const first_tree_attn_desc* d, int32_t B, int32_t N, int32_t max_nodes, int32_t max_len) {
  const int rc = tree_refusal(d, B, N, max_nodes, max_len);
  if (rc != FIRST_OK) return rc;
  const TreePlan p = tree_plan(*d, B, max_nodes, max_len);
  return p.splits == 1 ? 0 : 16 + (int64_t)p.splits * N * d->n_q_heads * (d->head_dim + 2) * 4;
}

int first_op_tree_attn(void* hip_stream, const first_tree_attn_desc* d, const void* q, const void* k_new, const void* v_new, const void* kv_layer,
                       const int32_t* page_table, const int32_t* lens, const int32_t* node_offsets, const uint64_t* tree_mask, void* out, float* lse, int32_t B,
                       int32_t N, int32_t max_nodes, int32_t max_len, void* workspace, int64_t workspace_bytes) {
  const int64_t need = first_op_tree_attn_workspace(d, B, N, max_nodes, max_len);
  if (need < 0) return (int)need;
  if (B == 0 || N == 0 || max_nodes == 0) return FIRST_OK;
  const bool cached = max_len > 0 && d->max_pages > 0;
  if (!q || !k_new || !v_new || !lens || !node_offsets || !out || (cached && (!kv_layer || !page_table)) || (need > 0 && !workspace))
    return refuse(FIRST_ERR_ARG, "first_op_tree_attn: null pointer");
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16) || !aligned(kv_layer, 16) || !aligned(page_table, 4) || !aligned(lens, 4) ||
      !aligned(node_offsets, 4) || !aligned(tree_mask, 8) || !aligned(lse, 4) || !aligned(workspace, 16))
    return refuse(FIRST_ERR_ARG, "first_op_tree_attn: a pointer is not aligned (16 bytes for q, k, v, out, the cache and the workspace)");
  if (tree_mask && (int64_t)d->mask_words * 64 < max_nodes) return refuse(FIRST_ERR_ARG, "first_op_tree_attn: mask_words * 64 is below max_nodes");
  if (workspace_bytes < need) return refuse(FIRST_ERR_CAPACITY, "first_op_tree_attn: the workspace is smaller than first_op_tree_attn_workspace says");
  const TreePlan p = tree_plan(*d, B, max_nodes, max_len);
  TreeArgs P = {q, k_new, v_new, kv_layer, page_table, lens, node_offsets, (const unsigned long long*)tree_mask, out, lse, B, N, d->n_q_heads, d->n_kv_heads, d->n_pages,
                cached ? d->max_pages : 0, d->mask_words, max_nodes, max_len, d->scale, p.split_keys, p.splits, p.places, p.step, p.block, nullptr, nullptr, nullptr};
  if (need > 0) {
    P.keys = (int*)workspace;
    P.part = (float*)workspace + 4;
    P.ml = P.part + (size_t)p.splits * N * d->n_q_heads * d->head_dim;
  }
  const hipStream_t st = stream_of(hip_stream);
  hipError_t e;
  if (d->dtype == FIRST_DTYPE_BF16) e = d->head_dim == 128 ? launch_tree<bf16, 128>(st, P, p) : launch_tree<bf16, 64>(st, P, p);
  else e = d->head_dim == 128 ? launch_tree<float, 128>(st, P, p) : launch_tree<float, 64>(st, P, p);
  return launched("first_op_tree_attn", e);
}

int64_t first_sample_workspace(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab < 1) return refuse(FIRST_ERR_ARG, "first_sample_workspace: negative rows, or vocab < 1");
  if (vocab > 1 << 30) return refuse(FIRST_ERR_CAPACITY, "first_sample: more than 2^30 tokens");
  return 0;
}

int first_sample(void* hip_stream, const float* logits, int64_t pitch, int32_t rows, int32_t vocab, const float* uniforms, const float* temperature,
                 const int32_t* top_k, const float* top_p, const float* min_p, int32_t* token_out, float* logprob_out, int32_t* kept_out, void* workspace,
                 int64_t workspace_bytes) {
  const int64_t need = first_sample_workspace(rows, vocab);
  if (need == FIRST_ERR_CAPACITY) return FIRST_ERR_CAPACITY;
  if (need < 0 || pitch < vocab || pitch > INT32_MAX) return refuse(FIRST_ERR_ARG, "first_sample: negative rows, vocab < 1, or a pitch below vocab or above 2^31 - 1");
  if (rows == 0) return FIRST_OK;
  if (!logits || !uniforms || !token_out || (need > 0 && !workspace)) return refuse(FIRST_ERR_ARG, "first_sample: null pointer");
  if (!aligned(logits, 4) || !aligned(uniforms, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(token_out, 4) ||
      !aligned(logprob_out, 4) || !aligned(kept_out, 4) || !aligned(workspace, 16))
    return refuse(FIRST_ERR_ARG, "first_sample: a pointer is not aligned (16 bytes for the workspace, 4 for the others)");
  if (workspace_bytes < need) return refuse(FIRST_ERR_CAPACITY, "first_sample: the workspace is smaller than first_sample_workspace says");
  int bits = 0;
  while (bits < 31 && (int64_t)1 << bits < vocab) ++bits;
  const int held = std::min(SR_HELD, (vocab / 4 + SR_THREADS - 1) / SR_THREADS);
  SampleArgs P = {logits, pitch, vocab, bits, std::min(50, 62 - bits), held, uniforms, temperature, top_k, top_p, min_p, token_out, logprob_out, kept_out};
  return launched("first_sample", launch<&k_sample_row>(stream_of(hip_stream), dim3(rows), SR_THREADS, (size_t)held * SR_THREADS * 16, P, (size_t)SR_HELD * SR_THREADS * 16));
}

}  // extern "C"
