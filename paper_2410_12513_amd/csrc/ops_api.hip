// C ABI of the operators of a step over drafted tokens (include/first.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
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
int launched(const char* name) noexcept {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return FIRST_OK;
  try { g_create_error = std::string(name) + ": " + hipGetErrorString(e); } catch (...) {}
  return FIRST_ERR_HIP;
}
bool known_type(int dtype) { return dtype == FIRST_DTYPE_FP32 || dtype == FIRST_DTYPE_BF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }
size_t size_of(int dtype) { return dtype == FIRST_DTYPE_BF16 ? 2 : 4; }
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

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
  for (int i = 0; i < d->rot_dim / 2; ++i) {
    const double f = std::exp(step * i);
    double g = f;
    if (d->scaling == FIRST_ROPE_LINEAR) g = f / d->factor;
    if (d->scaling == FIRST_ROPE_BANDS) {
      const double keep = std::min(1.0, std::max(0.0, (d->original_len * f / two_pi - d->low) / ((double)d->high - d->low)));
      g = (1.0 - keep) * f / d->factor + keep * f;
    }
    P.turns[i] = g / two_pi;
  }
  const dim3 grid((unsigned)rows);
  if (d->dtype == FIRST_DTYPE_BF16) hipLaunchKernelGGL(k_rope<bf16>, grid, dim3(WG), 0, stream_of(hip_stream), P);
  else hipLaunchKernelGGL(k_rope<float>, grid, dim3(WG), 0, stream_of(hip_stream), P);
  return launched("first_op_rope");
}

int64_t first_op_gemm_nt_lora_workspace(int32_t dtype, int32_t m, int32_t n, int32_t k, int32_t r) {
  if (!known_type(dtype) || m < 0 || n < 1 || k < 8 || k % 8 || r < 1 || r > LORA_RMAX)
    return refuse(FIRST_ERR_ARG, "first_op_gemm_nt_lora_workspace: unknown dtype, negative m, n < 1, k not a positive multiple of 8, or rank outside 1..64");
  return up((int64_t)m * up(r, 16) * 4, 256);
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
  if (m > 1 << 20) return refuse(FIRST_ERR_CAPACITY, "first_op_gemm_nt_lora: too many rows");
  LoraArgs P = {A, W, La, Lb, adapter, scale, C, (float*)workspace, m, n, k, r, (int)up(r, 16), n_adapters, accumulate != 0};
  const dim3 grid((n + 63) / 64, (m + 63) / 64);
  hipStream_t st = stream_of(hip_stream);
  if (dtype == FIRST_DTYPE_BF16) {
    hipLaunchKernelGGL(k_lora_shrink<bf16>, dim3(m), dim3(WG), 0, st, P);
    hipLaunchKernelGGL(k_lora_gemm<bf16>, grid, dim3(WG), 0, st, P);
  } else {
    hipLaunchKernelGGL(k_lora_shrink<float>, dim3(m), dim3(WG), 0, st, P);
    hipLaunchKernelGGL(k_lora_gemm<float>, grid, dim3(WG), 0, st, P);
  }
  return launched("first_op_gemm_nt_lora");
}

static int tree_refusal(const first_tree_attn_desc* d, int32_t B, int32_t N, int32_t max_nodes, int32_t max_len) {
  if (!d) return refuse(FIRST_ERR_ARG, "first_op_tree_attn: null description");
  if (!known_type(d->dtype) || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads % d->n_kv_heads || d->n_q_heads > 1024 || (d->head_dim != 64 && d->head_dim != 128) ||
      d->page_tokens != TREE_PAGE)
    return refuse(FIRST_ERR_ARG, "first_op_tree_attn: unknown dtype, heads outside 1..1024 or not a multiple of the KV heads, head_dim not 64 or 128, or pages not of 16 tokens");
  if (!std::isfinite(d->scale) || d->n_pages < 0 || d->max_pages < 0 || d->mask_words < 0)
    return refuse(FIRST_ERR_ARG, "first_op_tree_attn: scale not finite, or a negative size");
  if (B < 0 || N < 0 || max_nodes < 0 || max_len < 0) return refuse(FIRST_ERR_ARG, "first_op_tree_attn: a negative size");
  if (B > 65535) return refuse(FIRST_ERR_CAPACITY, "first_op_tree_attn: more than 65535 sequences");
  return FIRST_OK;
}

int64_t first_op_tree_attn_workspace(const first_tree_attn_desc* d, int32_t B, int32_t N, int32_t max_nodes, int32_t max_len) {
  const int rc = tree_refusal(d, B, N, max_nodes, max_len);
  return rc != FIRST_OK ? rc : 0;
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
  TreeArgs P = {q, k_new, v_new, kv_layer, page_table, lens, node_offsets, (const unsigned long long*)tree_mask, out, lse, B, N, d->n_q_heads, d->n_kv_heads, d->n_pages,
                cached ? d->max_pages : 0, d->mask_words, max_nodes, max_len, d->scale};
  const dim3 grid(max_nodes, d->n_q_heads, B);
  hipStream_t st = stream_of(hip_stream);
  if (d->dtype == FIRST_DTYPE_BF16) {
    if (d->head_dim == 128) hipLaunchKernelGGL((k_tree_rows<bf16, 128>), grid, dim3(WG), 0, st, P);
    else hipLaunchKernelGGL((k_tree_rows<bf16, 64>), grid, dim3(WG), 0, st, P);
  } else {
    if (d->head_dim == 128) hipLaunchKernelGGL((k_tree_rows<float, 128>), grid, dim3(WG), 0, st, P);
    else hipLaunchKernelGGL((k_tree_rows<float, 64>), grid, dim3(WG), 0, st, P);
  }
  return launched("first_op_tree_attn");
}

int64_t first_sample_workspace(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab < 1) return refuse(FIRST_ERR_ARG, "first_sample_workspace: negative rows, or vocab < 1");
  return 0;
}

int first_sample(void* hip_stream, const float* logits, int64_t pitch, int32_t rows, int32_t vocab, const float* uniforms, const float* temperature,
                 const int32_t* top_k, const float* top_p, const float* min_p, int32_t* token_out, float* logprob_out, int32_t* kept_out, void* workspace,
                 int64_t workspace_bytes) {
  const int64_t need = first_sample_workspace(rows, vocab);
  if (need < 0 || pitch < vocab || pitch > INT32_MAX) return refuse(FIRST_ERR_ARG, "first_sample: negative rows, vocab < 1, or a pitch below vocab or above 2^31 - 1");
  if (rows == 0) return FIRST_OK;
  if (!logits || !uniforms || !token_out || (need > 0 && !workspace)) return refuse(FIRST_ERR_ARG, "first_sample: null pointer");
  if (!aligned(logits, 4) || !aligned(uniforms, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(token_out, 4) ||
      !aligned(logprob_out, 4) || !aligned(kept_out, 4) || !aligned(workspace, 16))
    return refuse(FIRST_ERR_ARG, "first_sample: a pointer is not aligned (16 bytes for the workspace, 4 for the others)");
  if (workspace_bytes < need) return refuse(FIRST_ERR_CAPACITY, "first_sample: the workspace is smaller than first_sample_workspace says");
  int bits = 0;
  while (bits < 31 && (int64_t)1 << bits < vocab) ++bits;
  SampleArgs P = {logits, pitch, vocab, bits, std::min(50, 62 - bits), uniforms, temperature, top_k, top_p, min_p, token_out, logprob_out, kept_out};
  hipLaunchKernelGGL(k_sample_row, dim3(rows), dim3(SR_THREADS), 0, stream_of(hip_stream), P);
  return launched("first_sample");
}

}  // extern "C"
