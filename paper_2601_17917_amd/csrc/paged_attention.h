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
  int workers, parts, min_tiles;                   // how the key tiles are shared out (see the kernels)
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

size_t paged_attention_bf16_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block);
hipError_t launch_paged_attention_bf16(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream);

}  // namespace sdllm
