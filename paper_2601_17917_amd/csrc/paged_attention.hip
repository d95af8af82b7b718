// Attention over a paged K/V cache (sdllm_paged_attention): one wave per query row.  Visible keys are [0, sinks) and [lo, hi); a
// wave takes 64 of them at a time, a lane the score of one, then a lane the output columns.
#include "paged_attention.h"

namespace sdllm {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((unsigned)x << 16); }
__device__ __forceinline__ void store(float* p, float x) { *p = x; }
__device__ __forceinline__ void store(uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_attention_row_kernel(PagedArgs a) {
  __shared__ float q_s[4][D], p_s[4][64];
  __shared__ long long v_s[4][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long row = (long long)blockIdx.x * 4 + wave;
  if (row >= (long long)a.B * a.Hq * a.K) return;
  const int r = (int)(row % a.K);
  const int h = (int)(row / a.K % a.Hq), b = (int)(row / a.K / a.Hq);
  const int q_len = a.q_lens ? min(max(a.q_lens[b], 0), a.K) : a.K;
  if (r >= q_len) return;
  const int n = min(max(a.lens[b], 0), a.max_kv), N = n + (a.kb ? q_len : 0), kvh = h / a.g;
  const int p = N - q_len + r;
  const int hi = a.causal ? max(min(p + 1, N), 0) : N;
  const int lo = a.window ? min(max(p - a.window + 1, 0), hi) : 0;
  const int first = min(a.sinks, lo), count = first + hi - lo;
  const T* q = (const T*)a.q + b * a.q_st[0] + h * a.q_st[1] + r * a.q_st[2];
  for (int d = lane; d < D; d += 64) q_s[wave][d] = to_float(q[d]) * a.scale;
  float m = -3.0e38f, l = 0.f, o[D / 64];
#pragma unroll
  for (int u = 0; u < D / 64; ++u) o[u] = 0.f;
  for (int i0 = 0; i0 < count; i0 += 64) {
    const int i = i0 + lane;
    float s = -INFINITY;
    const T* vrow = nullptr;
    if (i < count) {
      const int key = i < first ? i : lo + i - first;
      const T* krow = nullptr;
      if (key < n) {
        const int page = a.table[(long long)b * a.max_pages + (key >> a.shift)];
        if ((unsigned)page < (unsigned)a.n_pages) {
          const long long at = ((((long long)page * a.Hkv + kvh) << a.shift) + (key & ((1 << a.shift) - 1))) * D;
          krow = (const T*)a.kp + at; vrow = (const T*)a.vp + at;
        }
      } else {
        krow = (const T*)a.kb + b * a.kb_st[0] + kvh * a.kb_st[1] + (key - n) * a.kb_st[2];
        vrow = (const T*)a.vb + b * a.vb_st[0] + kvh * a.vb_st[1] + (key - n) * a.vb_st[2];
      }
      if (krow) {
        s = 0.f;
        for (int d = 0; d < D; ++d) s = fmaf(q_s[wave][d], to_float(krow[d]), s);
      }
    }
    float mx = s;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    const float m_new = fmaxf(m, mx), corr = expf(m - m_new), w = expf(s - m_new);
    float sum = w;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    m = m_new;
    l = l * corr + sum;
#pragma unroll
    for (int u = 0; u < D / 64; ++u) o[u] *= corr;
    p_s[wave][lane] = w;
    v_s[wave][lane] = (long long)(uintptr_t)vrow;
    __builtin_amdgcn_wave_barrier();
    for (int j = 0; j < min(64, count - i0); ++j) {
      const T* vr = (const T*)(uintptr_t)v_s[wave][j];
      if (!vr) continue;
      const float w2 = p_s[wave][j];
#pragma unroll
      for (int u = 0; u < D / 64; ++u) o[u] = fmaf(w2, to_float(vr[lane + 64 * u]), o[u]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  T* out = (T*)a.out + b * a.o_st[0] + h * a.o_st[1] + r * a.o_st[2];
#pragma unroll
  for (int u = 0; u < D / 64; ++u) store(out + lane + 64 * u, l == 0.f ? 0.f : o[u] / l);
}

static bool few_rows(const sdllm_paged_attn_params& p) { return (long long)p.Hq / p.Hkv * p.K <= 32; }

size_t paged_attention_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  if (p.dtype == SDLLM_FP32) return 0;
  return few_rows(p) ? paged_stream_workspace_bytes(p, with_block) : paged_tile_workspace_bytes(p, with_block);
}

static void dense_or(const int64_t* given, int H, int K, int D, long long* out) {
  const bool dense = given[0] == 0 && given[1] == 0 && given[2] == 0;
  out[0] = dense ? (long long)H * K * D : given[0];
  out[1] = dense ? (long long)K * D : given[1];
  out[2] = dense ? D : given[2];
}

hipError_t launch_paged_attention(const sdllm_paged_attn_params& p, const void* q, const void* k_pages, const void* v_pages,
                                  const int32_t* table, const int32_t* lens, const void* k_block, const void* v_block,
                                  const int32_t* q_lens, void* out, void* workspace, hipStream_t stream) {
  PagedArgs a;
  a.q = q; a.kp = k_pages; a.vp = v_pages; a.table = table; a.lens = lens; a.kb = k_block; a.vb = v_block; a.q_lens = q_lens; a.out = out;
  dense_or(p.q_stride, p.Hq, p.K, p.D, a.q_st);
  dense_or(p.out_stride, p.Hq, p.K, p.D, a.o_st);
  dense_or(p.k_block_stride, p.Hkv, p.K, p.D, a.kb_st);
  dense_or(p.v_block_stride, p.Hkv, p.K, p.D, a.vb_st);
  a.B = p.B; a.Hq = p.Hq; a.Hkv = p.Hkv; a.g = p.Hq / p.Hkv; a.K = p.K; a.R = a.g * p.K; a.shift = __builtin_ctz(p.page_size); a.page_bytes = (unsigned)((long long)p.Hkv * p.page_size * p.D * 2);
  a.n_pages = p.n_pages; a.max_pages = p.max_pages; a.max_kv = p.max_kv_len; a.causal = p.causal; a.window = p.window; a.sinks = p.sinks;
  a.scale = p.scale > 0.f ? p.scale : 1.0f / sqrtf((float)p.D);
  a.scale_log2 = a.scale * kLog2e; a.thr8 = 8.0f / a.scale_log2;
  if (p.dtype == SDLLM_BF16) return few_rows(p) ? launch_paged_stream(p, a, workspace, stream) : launch_paged_tile(p, a, workspace, stream);
  const long long rows = (long long)p.B * p.Hq * p.K;
  const dim3 grid((unsigned)((rows + 3) / 4));
  if (p.D == 64) hipLaunchKernelGGL((paged_attention_row_kernel<float, 64>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_attention_row_kernel<float, 128>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sdllm
