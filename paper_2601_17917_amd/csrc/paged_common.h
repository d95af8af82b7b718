// Shared by the operators on a paged K/V cache (include/sdllm_paged.h).
#pragma once
#include "common.h"
#include "lds_dma.h"
#include "sdllm_paged.h"

namespace sdllm {

// Division of n < 2^31 by a constant 1 <= d < 2^31 with one high multiply (the round-up method of Granlund and Montgomery,
// "Division by invariant integers using multiplication", 1994: m = ceil(2^32 (2^s - d) / d), s = ceil(log2 d),
// q = (mulhi(n, m) + n) >> s; the sum stays below 2^32 because mulhi(n, m) <= n).
struct FastDiv {
  unsigned d = 1, m = 0, s = 0;
  FastDiv() = default;
  explicit FastDiv(unsigned div) : d(div) {
    while ((1ULL << s) < d) ++s;
    m = (unsigned)((((1ULL << s) - d) << 32) / d + 1);
  }
  __host__ __device__ unsigned div(unsigned n) const {
    return (unsigned)((((unsigned long long)n * m >> 32) + n) >> s);
  }
};

// Sum of a value over the lanes up to this one; all lanes active
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);       // row_shr:1, 2, 4, 8: sums within 16 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast:15, 31: and over them
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
}

// Strides of a tensor [B, H, K, D] as given, or the dense one's
inline void dense_or(const int64_t* given, int H, int K, int D, long long* out) {
  const bool dense = given[0] == 0 && given[1] == 0 && given[2] == 0;
  out[0] = dense ? (long long)H * K * D : given[0];
  out[1] = dense ? (long long)K * D : given[1];
  out[2] = dense ? D : given[2];
}

// Errors of entry points that live outside api.hip end up in the same per-thread text (sdllm_last_error)
int set_error(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

size_t paged_extend_workspace_bytes(const sdllm_paged_extend_params& p);
hipError_t launch_paged_extend(const sdllm_paged_extend_params& p, int32_t* table, const int32_t* lens, const int32_t* new_lens,
                               const uint8_t* do_append, const uint8_t* release, int32_t* free_pages, const int32_t* n_free,
                               int32_t* lens_out, int32_t* n_free_out, int32_t* slots, int32_t* granted, void* workspace,
                               hipStream_t stream);
hipError_t launch_paged_append(const sdllm_paged_append_params& p, void* k_pages, void* v_pages, const void* k_blocks,
                               const void* v_blocks, const int32_t* slots, hipStream_t stream);
hipError_t launch_qk_norm_rope(const sdllm_qk_norm_rope_params& p, const void* q, const void* k, const void* v,
                               const int32_t* positions, const void* q_weight, const void* k_weight, void* q_out, void* k_out,
                               void* k_pages, void* v_pages, const int32_t* slots, hipStream_t stream);
size_t paged_attention_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block);
hipError_t launch_paged_attention(const sdllm_paged_attn_params& p, const void* q, const void* k_pages, const void* v_pages,
                                  const int32_t* table, const int32_t* lens, const void* k_block, const void* v_block,
                                  const int32_t* q_lens, void* out, void* workspace, hipStream_t stream);

}  // namespace sdllm
