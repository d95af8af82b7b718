// Host side of the C ABI of include/sdllm_paged.h: argument validation (before any HIP call), workspace queries, dispatch.
#include "paged_common.h"
#include <cmath>

using sdllm::set_error;

namespace {

constexpr int kInvalid = SDLLM_ERR_INVALID_ARG, kUnsupported = SDLLM_ERR_UNSUPPORTED;

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_dtype(const char* what, int dtype) {
  if (dtype != SDLLM_FP32 && dtype != SDLLM_BF16) return set_error(kUnsupported, "%s: dtype %d not supported (fp32=0, bf16=1)", what, dtype);
  return SDLLM_OK;
}

int check_pages(const char* what, int page_size, int n_pages) {
  if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0)
    return set_error(kUnsupported, "%s: page_size %d not supported (a power of two, 16..1024)", what, page_size);
  if (n_pages < 1) return set_error(kInvalid, "%s: n_pages must be >= 1", what);
  if ((long long)n_pages * page_size > 0x7fffffffLL) return set_error(kUnsupported, "%s: n_pages * page_size must be below 2^31", what);
  return SDLLM_OK;
}

// Strides of a tensor [B, H, K, D] in elements; all zero: dense.  `written`: rows must not fall on one another.
int check_strides(const char* what, const char* name, const int64_t* s, long long B, long long H, long long K, long long D, int elem,
                  bool written) {
  if (s[0] == 0 && s[1] == 0 && s[2] == 0) return SDLLM_OK;
  for (int i = 0; i < 3; ++i) {
    if (s[i] < 0) return set_error(kInvalid, "%s: a stride of %s is negative", what, name);
    if (s[i] * elem % 16 != 0) return set_error(kInvalid, "%s: a stride of %s is not a multiple of 16 bytes", what, name);
    if (s[i] > (1LL << 40)) return set_error(kUnsupported, "%s: a stride of %s is too large", what, name);
  }
  if (!written) return SDLLM_OK;
  // sorted by stride, each dimension must step over everything that the smaller ones span
  const long long n[3] = {B, H, K};
  int o[3] = {0, 1, 2};
  for (int i = 0; i < 2; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (s[o[j]] < s[o[i]]) { const int x = o[i]; o[i] = o[j]; o[j] = x; }
  long long span = D;
  for (int i = 0; i < 3; ++i) {
    if (n[o[i]] == 1) continue;
    if (s[o[i]] < span) return set_error(kInvalid, "%s: rows of %s overlap", what, name);
    span += (n[o[i]] - 1) * s[o[i]];
  }
  return SDLLM_OK;
}

int check_extend(const sdllm_paged_extend_params* p) {
  if (!p) return set_error(kInvalid, "paged_extend: params is NULL");
  if (p->B < 1 || p->K < 1 || p->max_pages < 1) return set_error(kInvalid, "paged_extend: B, K, max_pages must be >= 1");
  if (int rc = check_pages("paged_extend", p->page_size, p->n_pages)) return rc;
  if (p->B > 65536 || (long long)p->B * p->K >= (1LL << 31) || (long long)p->B * p->max_pages >= (1LL << 30) ||
      (long long)p->max_pages * p->page_size > (1LL << 30) || p->K > (1 << 30))
    return set_error(kUnsupported, "paged_extend: batch, rows or tables too large");
  return SDLLM_OK;
}

int check_norm_rope(const sdllm_qk_norm_rope_params* p, bool paged) {
  const char* w = "qk_norm_rope";
  if (!p) return set_error(kInvalid, "%s: params is NULL", w);
  if (int rc = check_dtype(w, p->dtype)) return rc;
  if (p->B < 1 || p->K < 1 || p->Hq < 1 || p->Hkv < 1) return set_error(kInvalid, "%s: B, K, Hq, Hkv must be >= 1", w);
  if (p->D < 16 || p->D % 16 != 0 || p->D > 256) return set_error(kUnsupported, "%s: head_dim %d not supported (multiple of 16, <= 256)", w, p->D);
  if (p->rotary_dim < 0 || p->rotary_dim > p->D || p->rotary_dim % 16 != 0)
    return set_error(kInvalid, "%s: rotary_dim %d must be a multiple of 16 in 0..%d", w, p->rotary_dim, p->D);
  if (!(p->eps >= 0.f) || std::isinf(p->eps)) return set_error(kInvalid, "%s: eps must be finite and >= 0", w);
  if (!(p->theta_base > 1.0f) || std::isinf(p->theta_base)) return set_error(kInvalid, "%s: theta_base must be finite and > 1", w);
  if (!(p->scale_factor >= 1.0f) || std::isinf(p->scale_factor)) return set_error(kInvalid, "%s: scale_factor must be finite and >= 1", w);
  if (!(p->amplitude == p->amplitude) || std::isinf(p->amplitude)) return set_error(kInvalid, "%s: amplitude is not finite", w);
  if (p->original_len < 0) return set_error(kInvalid, "%s: original_len must be >= 0", w);
  if (p->original_len > 0 && (!(p->low_turns >= 0.f) || !(p->high_turns > p->low_turns) || std::isinf(p->high_turns)))
    return set_error(kInvalid, "%s: need 0 <= low_turns < high_turns", w);
  if (paged)
    if (int rc = check_pages(w, p->page_size, p->n_pages)) return rc;
  if ((long long)p->B * p->K > 0xffffffLL || p->Hq > 65535 || p->Hkv > 65535) return set_error(kUnsupported, "%s: problem too large", w);
  const int e = p->dtype == SDLLM_FP32 ? 4 : 2;
  if (int rc = check_strides(w, "q", p->q_stride, p->B, p->Hq, p->K, p->D, e, false)) return rc;
  if (int rc = check_strides(w, "k", p->k_stride, p->B, p->Hkv, p->K, p->D, e, false)) return rc;
  if (paged)
    if (int rc = check_strides(w, "v", p->v_stride, p->B, p->Hkv, p->K, p->D, e, false)) return rc;
  if (int rc = check_strides(w, "q_out", p->q_out_stride, p->B, p->Hq, p->K, p->D, e, true)) return rc;
  if (!paged)
    if (int rc = check_strides(w, "k_out", p->k_out_stride, p->B, p->Hkv, p->K, p->D, e, true)) return rc;
  return SDLLM_OK;
}

int check_paged_append(const sdllm_paged_append_params* p) {
  const char* w = "paged_kv_append";
  if (!p) return set_error(kInvalid, "%s: params is NULL", w);
  if (int rc = check_dtype(w, p->dtype)) return rc;
  if (p->n_layers < 1 || p->B < 1 || p->Hkv < 1 || p->D < 1 || p->K < 1) return set_error(kInvalid, "%s: n_layers, B, Hkv, D, K must be >= 1", w);
  if (int rc = check_pages(w, p->page_size, p->n_pages)) return rc;
  const int e = p->dtype == SDLLM_FP32 ? 4 : 2;
  if ((long long)p->D * e % 16 != 0) return set_error(kUnsupported, "%s: row size %lld bytes must be a multiple of 16", w, (long long)p->D * e);
  if (p->Hkv > 65535 || p->D > 65535) return set_error(kUnsupported, "%s: Hkv and D must be below 65536", w);
  // the products are formed step by step: each factor is below 2^31
  const long long rows = (long long)p->B * p->Hkv;
  if (rows > 0x7fffffffLL || rows * p->K > 0x7fffffffLL || rows * p->K * ((long long)p->D * e / 16) > 0x7fffffffLL)
    return set_error(kUnsupported, "%s: problem too large for one launch", w);
  const long long chunks = rows * p->K * ((long long)p->D * e / 16);
  if ((chunks + 1023) / 1024 * p->n_layers > 0xffffffLL) return set_error(kUnsupported, "%s: problem too large for one launch", w);
  const long long dense_p = (long long)p->n_pages * p->page_size * p->Hkv, dense_b = rows * p->K * p->D;
  if (p->pages_layer_stride != 0 && (p->pages_layer_stride / p->D < dense_p || p->pages_layer_stride * e % 16 != 0))
    return set_error(kInvalid, "%s: pages_layer_stride too small or not 16-byte aligned", w);
  if (p->block_layer_stride != 0 && (p->block_layer_stride < dense_b || p->block_layer_stride * e % 16 != 0))
    return set_error(kInvalid, "%s: block_layer_stride too small or not 16-byte aligned", w);
  return SDLLM_OK;
}

int check_paged_attn(const sdllm_paged_attn_params* p, bool with_block) {
  const char* w = "paged_attention";
  if (!p) return set_error(kInvalid, "%s: params is NULL", w);
  if (int rc = check_dtype(w, p->dtype)) return rc;
  if (p->B < 1 || p->Hq < 1 || p->Hkv < 1 || p->K < 1) return set_error(kInvalid, "%s: B, Hq, Hkv, K must be >= 1", w);
  if (p->Hq % p->Hkv != 0) return set_error(kInvalid, "%s: Hq (%d) must be a multiple of Hkv (%d)", w, p->Hq, p->Hkv);
  if (p->D != 64 && p->D != 128) return set_error(kUnsupported, "%s: head_dim %d not compiled (64, 128)", w, p->D);
  if (int rc = check_pages(w, p->page_size, p->n_pages)) return rc;
  if (p->max_pages < 1 || p->max_kv_len < 0 || p->max_kv_len > (long long)p->max_pages * p->page_size)
    return set_error(kInvalid, "%s: need max_pages >= 1 and 0 <= max_kv_len (%d) <= max_pages * page_size", w, p->max_kv_len);
  if (p->window < 0 || p->sinks < 0) return set_error(kInvalid, "%s: window and sinks must be >= 0", w);
  if (p->kv_splits < 0) return set_error(kInvalid, "%s: kv_splits must be >= 0", w);
  if (!(p->scale == p->scale) || std::isinf(p->scale)) return set_error(kInvalid, "%s: scale is not finite", w);
  if (p->scale > 1e38f) return set_error(kUnsupported, "%s: scale is too large", w);       // its product with log2 e is an fp32 number
  const long long rows = (long long)p->Hq * p->K;
  if ((long long)p->max_kv_len + p->K > (1LL << 30) || (long long)p->B * p->Hkv >= (1LL << 22) || rows >= (1LL << 28) ||
      rows * p->B >= (1LL << 28) || (long long)p->B * p->max_pages > 0x7fffffffLL)
    return set_error(kUnsupported, "%s: sequence or batch too large", w);
  const int e = p->dtype == SDLLM_FP32 ? 4 : 2;
  if ((long long)p->Hkv * p->page_size * p->D * e >= (1LL << 31)) return set_error(kUnsupported, "%s: a page of all heads must be below 2 GiB", w);
  if (int rc = check_strides(w, "q", p->q_stride, p->B, p->Hq, p->K, p->D, e, false)) return rc;
  if (int rc = check_strides(w, "out", p->out_stride, p->B, p->Hq, p->K, p->D, e, true)) return rc;
  if (with_block) {
    if (int rc = check_strides(w, "k_block", p->k_block_stride, p->B, p->Hkv, p->K, p->D, e, false)) return rc;
    if (int rc = check_strides(w, "v_block", p->v_block_stride, p->B, p->Hkv, p->K, p->D, e, false)) return rc;
  }
  return SDLLM_OK;
}

}  // namespace

extern "C" {

size_t sdllm_paged_extend_workspace_bytes(const sdllm_paged_extend_params* p) {
  if (check_extend(p) != SDLLM_OK) return (size_t)-1;
  return sdllm::paged_extend_workspace_bytes(*p);
}

int sdllm_paged_extend(const sdllm_paged_extend_params* p, int32_t* block_table, const int32_t* kv_lens, const int32_t* new_lens,
                       const uint8_t* do_append, const uint8_t* release, int32_t* free_pages, const int32_t* n_free,
                       int32_t* kv_lens_out, int32_t* n_free_out, int32_t* slots, int32_t* granted, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (int rc = check_extend(p)) return rc;
  if (!block_table || !kv_lens || !free_pages || !n_free || !kv_lens_out || !n_free_out || !slots || !granted)
    return set_error(kInvalid, "paged_extend: only new_lens, do_append and release may be NULL");
  const void* words[] = {block_table, kv_lens, new_lens, free_pages, n_free, kv_lens_out, n_free_out, slots, granted};
  for (const void* w : words)
    if (!aligned(w, 4)) return set_error(kInvalid, "paged_extend: an int32 pointer is not 4-byte aligned");
  const size_t need = sdllm::paged_extend_workspace_bytes(*p);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return set_error(SDLLM_ERR_WORKSPACE, "paged_extend: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  if (need > 0 && !aligned(workspace, 16)) return set_error(kInvalid, "paged_extend: workspace is not 16-byte aligned");
  hipError_t e = sdllm::launch_paged_extend(*p, block_table, kv_lens, new_lens, do_append, release, free_pages, n_free, kv_lens_out,
                                            n_free_out, slots, granted, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SDLLM_ERR_HIP, "paged_extend: %s", hipGetErrorString(e));
  return SDLLM_OK;
}

int sdllm_qk_norm_rope(const sdllm_qk_norm_rope_params* p, const void* q, const void* k, const void* v, const int32_t* positions,
                       const void* q_weight, const void* k_weight, void* q_out, void* k_out, void* k_pages, void* v_pages,
                       const int32_t* slots, void* stream) {
  const bool paged = slots != nullptr;
  if (int rc = check_norm_rope(p, paged)) return rc;
  if (!q || !k || !positions || !q_out) return set_error(kInvalid, "qk_norm_rope: q, k, positions, q_out must not be NULL");
  if (paged ? (!v || !k_pages || !v_pages || k_out) : (!k_out || v || k_pages || v_pages))
    return set_error(kInvalid, "qk_norm_rope: give either k_out, or v, k_pages, v_pages and slots");
  const void* ptrs[] = {q, k, v, q_weight, k_weight, q_out, k_out, k_pages, v_pages};
  for (const void* x : ptrs)
    if (!aligned(x, 16)) return set_error(kInvalid, "qk_norm_rope: a base pointer is not 16-byte aligned");
  if (!aligned(positions, 4) || !aligned(slots, 4)) return set_error(kInvalid, "qk_norm_rope: positions / slots is not 4-byte aligned");
  hipError_t e = sdllm::launch_qk_norm_rope(*p, q, k, v, positions, q_weight, k_weight, q_out, k_out, k_pages, v_pages, slots,
                                            (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SDLLM_ERR_HIP, "qk_norm_rope: %s", hipGetErrorString(e));
  return SDLLM_OK;
}

int sdllm_paged_kv_append(const sdllm_paged_append_params* p, void* k_pages, void* v_pages, const void* k_blocks,
                          const void* v_blocks, const int32_t* slots, void* stream) {
  if (int rc = check_paged_append(p)) return rc;
  if (!k_pages || !v_pages || !k_blocks || !v_blocks || !slots) return set_error(kInvalid, "paged_kv_append: pages, blocks and slots must not be NULL");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(k_blocks, 16) || !aligned(v_blocks, 16) || !aligned(slots, 4))
    return set_error(kInvalid, "paged_kv_append: a base pointer is not 16-byte aligned (slots: 4)");
  hipError_t e = sdllm::launch_paged_append(*p, k_pages, v_pages, k_blocks, v_blocks, slots, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SDLLM_ERR_HIP, "paged_kv_append: %s", hipGetErrorString(e));
  return SDLLM_OK;
}

size_t sdllm_paged_attention_workspace_bytes(const sdllm_paged_attn_params* p, int32_t with_block) {
  if (check_paged_attn(p, with_block != 0) != SDLLM_OK) return (size_t)-1;
  return sdllm::paged_attention_workspace_bytes(*p, with_block != 0);
}

int sdllm_paged_attention(const sdllm_paged_attn_params* p, const void* q, const void* k_pages, const void* v_pages,
                          const int32_t* block_table, const int32_t* kv_lens, const void* k_block, const void* v_block,
                          const int32_t* q_lens, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const bool with_block = k_block != nullptr;
  if (int rc = check_paged_attn(p, with_block)) return rc;
  if (!q || !k_pages || !v_pages || !block_table || !kv_lens || !out)
    return set_error(kInvalid, "paged_attention: q, k_pages, v_pages, block_table, kv_lens, out must not be NULL");
  if (with_block != (v_block != nullptr)) return set_error(kInvalid, "paged_attention: give both of k_block and v_block, or neither");
  const void* ptrs[] = {q, k_pages, v_pages, k_block, v_block, out};
  for (const void* x : ptrs)
    if (!aligned(x, 16)) return set_error(kInvalid, "paged_attention: a base pointer is not 16-byte aligned");
  if (!aligned(block_table, 4) || !aligned(kv_lens, 4) || !aligned(q_lens, 4))
    return set_error(kInvalid, "paged_attention: an int32 pointer is not 4-byte aligned");
  const size_t need = sdllm::paged_attention_workspace_bytes(*p, with_block);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return set_error(SDLLM_ERR_WORKSPACE, "paged_attention: workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  if (need > 0 && !aligned(workspace, 16)) return set_error(kInvalid, "paged_attention: workspace is not 16-byte aligned");
  hipError_t e = sdllm::launch_paged_attention(*p, q, k_pages, v_pages, block_table, kv_lens, k_block, v_block, q_lens, out,
                                               need ? workspace : nullptr, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(SDLLM_ERR_HIP, "paged_attention: %s", hipGetErrorString(e));
  return SDLLM_OK;
}

}  // extern "C"
