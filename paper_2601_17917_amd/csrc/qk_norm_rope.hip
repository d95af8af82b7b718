// Norms of queries and keys for each head and the position rotation in one pass over the rows (sdllm_qk_norm_rope), the keys
// and values optionally straight into their pages.
//     y = x / sqrt(mean(x^2) + eps) * w;   (y_a, y_b) -> amplitude * (y_a cos - y_b sin, y_b cos + y_a sin)
// One read and one write of every row: bound by HBM, or for few rows by the launch and two round trips.
//
// A workgroup takes one token and a chunk of its heads.  The token's cos / sin are computed once per workgroup: the angle in
// turns, position * f_i / 2 pi, in double (its fraction is what counts, and float loses it beyond a few thousand positions), the
// fraction's sine and cosine in float.  A lane holds two 16-byte vectors of a row that contain whole pairs -- (i, i + R/2) as a
// vector of the first half and the matching one of the second, or adjacent vectors -- so that the rotation needs no exchange
// between lanes; the sum of squares is reduced over the 4 to 32 lanes of a row.  2 x 4096 tokens of 36 heads of 128, 151 MB,
// take 25 us (6.1 TB/s); several tokens for a workgroup were slower (36 to 42 where one each took 33, before outputs went past L2).
#include "paged_common.h"
#include <cmath>

namespace sdllm {

constexpr int kMaxPairs = 128;

struct NormRopeArgs {
  const void* q; const void* k; const void* v; const int32_t* positions; const void* qw; const void* kw;
  void* q_out; void* k_out; void* k_pages; void* v_pages; const int32_t* slots;
  long long q_st[3], k_st[3], v_st[3], qo_st[3], ko_st[3];   // elements
  int K, Hq, Hkv, rows, rows_per_chunk;                      // rows: heads of a token over q, k and, with pages, v
  int D, R, per_row, shift, slots_total;
  float eps, amplitude;
  double turns[kMaxPairs];                                   // turns per position of each pair
};

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void unpack(const u32x4& r, float* x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(r[e]);
  }
  __device__ static __forceinline__ u32x4 pack(const float* x) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};
template <> struct Vec<uint16_t> {                           // bf16 bit patterns, rounded to nearest even
  static constexpr int N = 8;
  __device__ static __forceinline__ void unpack(const u32x4& r, float* x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(r[e] << 16); x[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u); }
  }
  __device__ static __forceinline__ u32x4 pack(const float* x) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x[2 * e], x[2 * e + 1]}, bf16x2));
    return r;
  }
};

// GL lanes per row (a power of two, at least D / (2 N); the lanes beyond idle)
template <typename T, int GL, bool INTERLEAVED, bool STREAMING>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(NormRopeArgs a) {
  constexpr int N = Vec<T>::N;
  __shared__ float cos_s[kMaxPairs], sin_s[kMaxPairs];
  const int tid = threadIdx.x;
  const int token = blockIdx.x;
  const int b = token / a.K, t = token - b * a.K;

  const int j = tid % GL;
  const bool active = j < a.D / (2 * N);
  // the lane's two vectors of a row
  const int half = a.R / (2 * N);
  const bool turned = INTERLEAVED ? 2 * j < a.R / N : j < half;
  int va, vb;
  if (INTERLEAVED || !turned) { va = INTERLEAVED ? 2 * j : a.R / N + 2 * (j - half); vb = va + 1; }
  else { va = j; vb = j + half; }
  const int first = INTERLEAVED ? j * N : va * N;            // its first pair

  const int row0 = blockIdx.y * a.rows_per_chunk, row1 = min(row0 + a.rows_per_chunk, a.rows);
  u32x4 na{}, nb{};                                // a row's loads travel under the angles, or under the row before
  auto load = [&](int row) {
    if (row >= row1 || !active) return;
    const bool is_q = row < a.Hq, is_v = row >= a.Hq + a.Hkv;
    const int h = is_q ? row : (is_v ? row - a.Hq - a.Hkv : row - a.Hq);
    const long long* st = is_q ? a.q_st : (is_v ? a.v_st : a.k_st);
    const T* src = (const T*)(is_q ? a.q : (is_v ? a.v : a.k)) + b * st[0] + h * st[1] + t * st[2];
    na = *reinterpret_cast<const u32x4*>(src + va * N);
    nb = *reinterpret_cast<const u32x4*>(src + vb * N);
  };
  load(row0 + tid / GL);
  for (int i = tid; i < a.R / 2; i += 256) {
    const double pos = a.per_row ? (double)a.positions[token] : (double)a.positions[b] + t;    // a sum may pass 2^31
    const double x = pos * a.turns[i];
    const float r = (float)(x - rint(x));
    float s, c;
    sincospif(2.0f * r, &s, &c);
    cos_s[i] = c * a.amplitude; sin_s[i] = s * a.amplitude;
  }
  const int slot = a.slots != nullptr ? a.slots[token] : -1;
  __syncthreads();

  for (int row = row0 + tid / GL; row < row1; row += 256 / GL) {
    // which tensor: uniform over the lanes of a row
    const bool is_q = row < a.Hq, is_v = row >= a.Hq + a.Hkv;
    const int h = is_q ? row : (is_v ? row - a.Hq - a.Hkv : row - a.Hq);
    const u32x4 ra = na, rb = nb;
    load(row + 256 / GL);
    T* dst;
    if (is_q) dst = (T*)a.q_out + b * a.qo_st[0] + h * a.qo_st[1] + t * a.qo_st[2];
    else if (a.slots == nullptr) dst = (T*)a.k_out + b * a.ko_st[0] + h * a.ko_st[1] + t * a.ko_st[2];
    else {
      if ((unsigned)slot >= (unsigned)a.slots_total) continue;
      const int page = slot >> a.shift, r = slot & ((1 << a.shift) - 1);
      dst = (T*)(is_v ? a.v_pages : a.k_pages) + ((((long long)page * a.Hkv + h) << a.shift) + r) * a.D;
    }
    auto store = [&](const u32x4& x, const u32x4& y) {
      u32x4 *to = reinterpret_cast<u32x4*>(dst + va * N), *to2 = reinterpret_cast<u32x4*>(dst + vb * N);
      if constexpr (STREAMING) { __builtin_nontemporal_store(x, to); __builtin_nontemporal_store(y, to2); }
      else { *to = x; *to2 = y; }
    };
    if (is_v) {
      if (active) store(ra, rb);
      continue;
    }
    float x[2 * N];
    Vec<T>::unpack(ra, x); Vec<T>::unpack(rb, x + N);
    const T* w = (const T*)(is_q ? a.qw : a.kw);
    if (w != nullptr) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int d = 1; d < GL; d <<= 1) ss += __shfl_xor(ss, d);
      const float inv = rsqrtf(ss / (float)a.D + a.eps);
      if (active) {
        float wf[2 * N];
        Vec<T>::unpack(*reinterpret_cast<const u32x4*>(w + va * N), wf);
        Vec<T>::unpack(*reinterpret_cast<const u32x4*>(w + vb * N), wf + N);
#pragma unroll
        for (int e = 0; e < 2 * N; ++e) x[e] = x[e] * inv * wf[e];
      }
    }
    if (!active) continue;
    if (turned) {
      float y[2 * N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int ia = INTERLEAVED ? 2 * e : e, ib = INTERLEAVED ? 2 * e + 1 : e + N;
        const float c = cos_s[first + e], s = sin_s[first + e];
        y[ia] = x[ia] * c - x[ib] * s;
        y[ib] = x[ib] * c + x[ia] * s;
      }
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) x[e] = y[e];
    }
    store(Vec<T>::pack(x), Vec<T>::pack(x + N));
  }
}

template <typename T, int GL>
static void launch_gl(const NormRopeArgs& a, bool interleaved, bool streaming, dim3 grid, hipStream_t stream) {
  if (interleaved) {
    if (streaming) hipLaunchKernelGGL((qk_norm_rope_kernel<T, GL, true, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<T, GL, true, false>), grid, dim3(256), 0, stream, a);
  } else {
    if (streaming) hipLaunchKernelGGL((qk_norm_rope_kernel<T, GL, false, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<T, GL, false, false>), grid, dim3(256), 0, stream, a);
  }
}

hipError_t launch_qk_norm_rope(const sdllm_qk_norm_rope_params& p, const void* q, const void* k, const void* v,
                               const int32_t* positions, const void* q_weight, const void* k_weight, void* q_out, void* k_out,
                               void* k_pages, void* v_pages, const int32_t* slots, hipStream_t stream) {
  NormRopeArgs a;
  a.q = q; a.k = k; a.v = v; a.positions = positions; a.qw = q_weight; a.kw = k_weight;
  a.q_out = q_out; a.k_out = k_out; a.k_pages = k_pages; a.v_pages = v_pages; a.slots = slots;
  dense_or(p.q_stride, p.Hq, p.K, p.D, a.q_st);
  dense_or(p.k_stride, p.Hkv, p.K, p.D, a.k_st);
  dense_or(p.v_stride, p.Hkv, p.K, p.D, a.v_st);
  dense_or(p.q_out_stride, p.Hq, p.K, p.D, a.qo_st);
  dense_or(p.k_out_stride, p.Hkv, p.K, p.D, a.ko_st);
  a.K = p.K; a.Hq = p.Hq; a.Hkv = p.Hkv; a.D = p.D; a.R = p.rotary_dim; a.per_row = p.positions_per_row;
  a.shift = slots ? __builtin_ctz(p.page_size) : 0;
  a.slots_total = slots ? p.n_pages << a.shift : 0;
  // What is more than the L2s hold is not kept there for the reader.  (Three sets of tensors in turn, past L2
  // and through it: 2 x 4096 tokens of 36 heads of 128 26.6 us and 33.8, 2 x 4000 of 48 heads of 64 18.6 and 24.3.)
  const bool streaming = (double)p.B * p.K * (p.Hq + p.Hkv * (slots ? 2 : 1)) * p.D * (p.dtype == SDLLM_FP32 ? 4 : 2) > 32e6;
  a.eps = p.eps; a.amplitude = p.amplitude;
  a.rows = p.Hq + p.Hkv * (slots ? 2 : 1);
  // turns per position of pair i: theta^(-2i/R) / 2 pi, by repeated multiplication (64 roundings of 2^-53)
  const double step = p.rotary_dim ? std::exp2(-2.0 / p.rotary_dim * std::log2((double)p.theta_base)) : 1.0;
  const double s = p.scale_factor;
  double f = 1.0 / (2.0 * M_PI);
  for (int i = 0; i < p.rotary_dim / 2; ++i, f *= step) {
    double u = 0.0;
    if (p.original_len > 0) u = std::fmin(std::fmax((f * p.original_len - p.low_turns) / ((double)p.high_turns - p.low_turns), 0.0), 1.0);
    a.turns[i] = s == 1.0 ? f : u * f + (1.0 - u) * f / s;
  }
  const bool f32 = p.dtype == SDLLM_FP32;
  const int lanes = p.D / (f32 ? 8 : 16);
  int gl = 4;
  while (gl < lanes) gl *= 2;
  // heads of a token in one workgroup, but enough workgroups to fill the chip where there are few tokens
  const long long tokens = (long long)p.B * p.K;
  const int per_pass = 256 / gl;
  long long chunks = (2 * kNumCUs + tokens - 1) / tokens;
  const int most = (a.rows + per_pass - 1) / per_pass;
  if (chunks > most) chunks = most;
  a.rows_per_chunk = (int)((a.rows + chunks - 1) / chunks);
  chunks = (a.rows + a.rows_per_chunk - 1) / a.rows_per_chunk;
  const dim3 grid((unsigned)tokens, (unsigned)chunks);
  const bool il = p.interleaved != 0;
  if (f32) {
    if (gl == 4) launch_gl<float, 4>(a, il, streaming, grid, stream);
    else if (gl == 8) launch_gl<float, 8>(a, il, streaming, grid, stream);
    else if (gl == 16) launch_gl<float, 16>(a, il, streaming, grid, stream);
    else launch_gl<float, 32>(a, il, streaming, grid, stream);
  } else {
    if (gl == 4) launch_gl<uint16_t, 4>(a, il, streaming, grid, stream);
    else if (gl == 8) launch_gl<uint16_t, 8>(a, il, streaming, grid, stream);
    else launch_gl<uint16_t, 16>(a, il, streaming, grid, stream);
  }
  return hipGetLastError();
}

}  // namespace sdllm
