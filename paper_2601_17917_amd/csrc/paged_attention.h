// Shared by the kernels of sdllm_paged_attention.
#pragma once
#include "paged_common.h"

namespace sdllm {

struct PagedArgs {
  const void* q; const void* kp; const void* vp; const int32_t* table; const int32_t* lens;
  const void* kb; const void* vb; const int32_t* q_lens; void* out;
  float* ws_o; float* ws_ml;                       // partial results: unnormalised output rows, (reference score, sum)
  long long q_st[3], o_st[3], kb_st[3], vb_st[3];  // elements
  int B, Hq, Hkv, g, K, R;                         // R = g K: query rows of a (sequence, K/V head)
  int shift, n_pages, max_pages, max_kv, causal, window, sinks;
  int workers, parts, row_tiles, min_tiles;        // how the key tiles are shared out (see the kernels)
  float scale, scale_log2, thr8;                    // thr8: 8 in log2 units, as a difference of scores
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegBig = -3.0e38f;

// Query row R of a (sequence, K/V head): row r = R / g of query head kvh g + R % g.  The heads that share K/V lie side by side, so
// that a tile of query rows spans few positions (few keys under a causal mask or a window) and the rows of a short sequence are
// the first ones.

// What a tile of query rows [r0, r1] of a sequence sees: keys [0, sink) and [lo, hi) of N, in tiles of TK keys:
// tile index i < sink_tiles is key tile i, the others follow from key tile first on.
struct Seen {
  int n, q_len, N;                                 // cached rows, query rows, keys
  int p0, p1;                                      // positions of the first and the last row
  int lo, hi, sink;
  int sink_tiles, first, tiles;
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : first + i - sink_tiles; }
};

__device__ __forceinline__ Seen seen_by(const PagedArgs& a, int n, int q_len, int r0, int r1, int TK) {
  Seen s;
  s.n = min(max(n, 0), a.max_kv);
  s.q_len = min(max(q_len, 0), a.K);
  s.N = s.n + (a.kb != nullptr ? s.q_len : 0);
  s.p0 = s.N - s.q_len + r0;
  s.p1 = s.N - s.q_len + min(r1, s.q_len - 1);
  s.hi = a.causal ? min(max(s.p1 + 1, 0), s.N) : s.N;
  s.lo = a.window > 0 ? min(max(s.p0 - a.window + 1, 0), s.hi) : 0;
  s.sink = min(a.sinks, s.lo);
  s.first = s.lo / TK;
  s.sink_tiles = min((s.sink + TK - 1) / TK, s.first);
  s.tiles = s.sink_tiles + (s.hi + TK - 1) / TK - s.first;       // lo < hi unless both are 0: then none
  return s;
}

// Keys visible to row r of the tile: [lo, hi) and below sinks
__device__ __forceinline__ void row_range(const PagedArgs& a, const Seen& s, int r, int& lo, int& hi) {
  const int p = s.N - s.q_len + r;
  hi = a.causal ? min(max(p + 1, 0), s.N) : s.N;
  lo = a.window > 0 ? max(p - a.window + 1, 0) : 0;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Everything in front of these is done before anything behind them: transfers have landed, LDS reads are in registers.  (The
// waits are the builtin, which the compiler's own wait insertion takes into account; the empty statements keep it from moving
// memory accesses across.)
__device__ __forceinline__ void wait_transfers() {
  asm volatile("" ::: "memory");
  wait_vmcnt<0>();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// Key tiles of each sequence (over one K/V head), and the sum over the batch.  The lanes take 64 sequences at a time.
template <int TK>
__device__ __forceinline__ int tiles_of(const PagedArgs& a, int b) {
  if (b >= a.B) return 0;
  const Seen s = seen_by(a, a.lens[b], a.q_lens ? a.q_lens[b] : a.K, 0, a.K - 1, TK);
  return s.q_len > 0 ? max(s.tiles, 1) : 0;        // rows that see nothing are a tile of their own: they are zero
}
__device__ __forceinline__ int wave_scan(int v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(v, d);
    if ((int)(threadIdx.x & 63) >= d) v += up;
  }
  return v;
}
template <int TK>
__device__ __forceinline__ long long all_tiles(const PagedArgs& a) {
  long long total = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) total += uniform(__shfl(wave_scan(tiles_of<TK>(a, b0 + (int)(threadIdx.x & 63))), 63));
  return total * a.Hkv;
}
__device__ __forceinline__ long long tiles_per_worker(const PagedArgs& a, long long total) {
  const long long n = (total + a.workers - 1) / a.workers;
  return n > a.min_tiles ? n : a.min_tiles;
}

// A (sequence, K/V head) being walked; everything uniform
struct Unit {
  int b, kvh, i, T;                                // tile i of T
  Seen s;
};

template <int TK>
__device__ __forceinline__ void open_unit(const PagedArgs& a, Unit& u, int b, int kvh, int i) {
  u.b = b; u.kvh = kvh; u.i = i;
  const const_i32_ptr lens = (const_i32_ptr)(uintptr_t)a.lens, q_lens = (const_i32_ptr)(uintptr_t)a.q_lens;
  u.s = seen_by(a, lens[b], a.q_lens ? q_lens[b] : a.K, 0, a.K - 1, TK);
  u.T = u.s.q_len > 0 ? max(u.s.tiles, 1) : 0;
}

// The unit and tile at position f of the call's tiles
template <int TK>
__device__ __forceinline__ void locate(const PagedArgs& a, long long f, Unit& u) {
  const int lane = threadIdx.x & 63;
  long long before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int t = tiles_of<TK>(a, b0 + lane), upto = wave_scan(t);
    const int chunk = uniform(__shfl(upto, 63));
    if (f < before + (long long)chunk * a.Hkv) {
      const unsigned long long above = __ballot((long long)upto * a.Hkv > f - before);
      const int l = __builtin_ctzll(above);
      const int tb = uniform(__shfl(t, l)), first = uniform(__shfl(upto, l)) - tb;
      const long long rest = f - before - (long long)first * a.Hkv;
      const int kvh = (int)(rest / tb);
      open_unit<TK>(a, u, b0 + l, kvh, (int)(rest - (long long)kvh * tb));
      return;
    }
    before += (long long)chunk * a.Hkv;
  }
}
template <int TK>
__device__ __forceinline__ void next_tile(const PagedArgs& a, Unit& u) {
  if (++u.i < u.T) return;
  if (u.kvh + 1 < a.Hkv) { ++u.kvh; u.i = 0; return; }
  int b = u.b;
  do { open_unit<TK>(a, u, ++b, 0, 0); } while (u.T == 0 && b + 1 < a.B);
}

// Values that are not finite, in a tile whose keys some rows see and others do not: a weight of 0 times such a value would be NaN
// in the rows that do not see it.  They are taken out of the product (0), and their effect on the rows that see them -- +inf, -inf,
// NaN -- is found from products of 0 / 1 matrices: which rows see which keys, which keys hold such a value in a column.
__device__ __forceinline__ bool has_nonfinite(const u32x4& x) {      // eight bf16
  bool bad = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) bad |= ((x[w] & 0x7f80u) == 0x7f80u) | ((x[w] & 0x7f800000u) == 0x7f800000u);
  return bad;
}
__device__ __forceinline__ s16x8 finite_part(const s16x8& v) { return ((v & (short)0x7f80) == (short)0x7f80) ? s16x8(0) : v; }
// 1 where v is +inf (kind 0), -inf (1), NaN (2); kind is uniform
__device__ __forceinline__ s16x8 is_kind(const s16x8& v, int kind) {
  const s16x8 nan = (v & (short)0x7fff) > (short)0x7f80, inf = v == (short)(kind == 0 ? 0x7f80 : 0xff80);
  return (kind == 2 ? nan : inf) & (short)0x3f80;
}
__device__ __forceinline__ float of_kind(int kind) { return kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __builtin_nanf(""); }
// 1 where a weight is not zero
__device__ __forceinline__ s16x8 weighed(const s16x8& p) { return p != 0 ? s16x8(0x3f80) : s16x8(0); }

// Kernels by query rows per (sequence, K/V head): up to 32 (stream), more (tile); both bf16
size_t paged_stream_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block);
hipError_t launch_paged_stream(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream);
size_t paged_tile_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block);
hipError_t launch_paged_tile(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream);
hipError_t launch_shares_merge(const PagedArgs& a, int D, int TK, hipStream_t stream);

}  // namespace sdllm
