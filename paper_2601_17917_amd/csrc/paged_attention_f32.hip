// fp32 attention over a paged K/V cache (sdllm_paged_attention) on the matrix cores (v_mfma_f32_16x16x4_f32).
//
// A unit is 16 query rows of a (sequence, K/V head).  Every wave walks a contiguous share of all units' 16-key tiles, laid end to end
// as in the bf16 stream kernel, or the eight waves of a workgroup share one unit (TOGETHER); K and V go from memory straight into
// registers in operand layout, without LDS or barriers.  The
// contraction index and the output column of a matrix instruction may be numbered at will as long as both sides agree:
//   S^T = K Q^T: step (c, e) multiplies d = 16 c + 4 G + e, so that a lane loads 16 bytes of a row of K (and of Q) at a time;
//   O^T = V^T P^T: step r multiplies keys 4 G + r, where the accumulators of S^T already hold P; row i of output block (c, b) is
//         column d = 64 c + 4 i + b, so that 16 bytes of V serve four blocks and a lane ends up with 16 columns in a row.
// Sums, weights and products stay in fp32 throughout.  Few rows and short spans are latency, not bandwidth: 4 sequences, 16 and 4 heads
// of 64, 5 query rows with a window of 1024 and 4 sinks (6.9 MB of K/V), take 17 us with the merge; a wave per query
// row with scalar products took 320 us.
#include "paged_attention.h"

namespace sdllm {

// global addresses as such: a pointer that the compiler knows nothing about would be read with flat loads, which wait for LDS, too
typedef const float __attribute__((address_space(1))) * global_ptr;
typedef const f32x4 __attribute__((address_space(1))) * vec_ptr;
__device__ __forceinline__ global_ptr rows_at(const void* base, long long byte) { return (global_ptr)((uintptr_t)base + byte); }

template <int D, bool TOGETHER>
__global__ __launch_bounds__(TOGETHER ? 512 : 256, 2) void paged_f32_kernel(PagedArgs) {
  constexpr int NW = TOGETHER ? 8 : 4, TK = 16, NC = D / 16, NV = D / 64;
  const int lane = threadIdx.x & 63, l16 = lane & 15, G = lane >> 4;
  extern __shared__ __attribute__((aligned(16))) float part_s[];       // TOGETHER: (rows of D, then reference and sum) of each wave
  const int wave = uniform(threadIdx.x >> 6), worker = TOGETHER ? blockIdx.x : blockIdx.x * NW + wave;
  const Hot h = hot_arguments();
  Pages pages;
  Unit cur;
  int left;
  {
    const Args a = arguments();
    if (worker >= a->workers) return;
    if (a->min_tiles == 0) {
      open_whole_unit<TK>(cur, pages, h, worker);
      left = cur.T;
    } else {
      left = open_share<TK>(worker, cur);
      pages.open(cur.b);
    }
  }
  [[maybe_unused]] int waves = 0;                  // of the workgroup that have tiles
  if constexpr (TOGETHER) {
    const int per = (left + NW - 1) / NW;
    if (left == 0) return;
    waves = (left + per - 1) / per;
    cur.i = wave * per;
    left = min(per, left - cur.i);
    if (left <= 0) {
      if (waves > 1) {                             // the barrier that the waves with tiles come to
        __syncthreads();
        merge_waves<float, D, 64 * NW>(cur, cur.rt * 16, 16, waves, part_s, 16 * D, part_s + NW * 16 * D, 32);
      }
      return;
    }
  }
  if (left == 0) return;
  int part = 0;
  while (left > 0) {
    const int begin = cur.i;
    f32x4 q[NC];
    int lo, hi, all_hi, all_lo, row0;
    global_ptr dummy;                              // a row that exists, for keys that do not
    {
      const Args a = arguments();
      const int g = a->g, last_row = cur.s.q_len * g - 1;
      row0 = cur.rt * 16;
      const int R = min(row0 + l16, last_row), r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
      const float* qp = (const float*)a->q + cur.b * a->q_st[0] + hq * a->q_st[1] + r * a->q_st[2];
      dummy = rows_at(qp, 0);
#pragma unroll
      for (int c = 0; c < NC; ++c) q[c] = *(vec_ptr)(dummy + 16 * c + 4 * G);
      row_range(a, cur.s, r, lo, hi);
      all_hi = a->causal ? cur.s.p0 + 1 : 0x7fffffff;
      all_lo = a->window > 0 ? cur.s.p1 - a->window + 1 : 0;
    }
    f32x4 o[NV][4];
    float m = kNegBig, limit = kNegBig, lsum = 0.f;   // reference of the weights; the score that moves it
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
      for (int b = 0; b < 4; ++b) o[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Loads of a tile's K, and of the V of the tile whose K was loaded last; a row of K or V that no query row sees, or that is not
    // there, is not read (bit j of vis: key j of the tile is seen).
    const Seen& s = cur.s;
    f32x4 k[NC], v[4][NV];
    auto load_k = [&](int i) -> unsigned {
      if (s.tiles == 0) return 0;
      const int k0 = s.tile(i) * TK;
      pages.seek(h, k0);
      const global_ptr page = rows_at(h.kp, row_offset(h, pages.of(h, k0), cur.kvh, k0, 4 * D));
      if (pages.ok(h, k0) && ((k0 >= s.lo && k0 <= s.last16) || k0 <= s.sink16)) {
#pragma unroll
        for (int c = 0; c < NC; ++c) k[c] = *(vec_ptr)(page + l16 * D + 16 * c + 4 * G);
        return 0xffffu;
      }
      // a border of what is seen, the end of the cache, rows of the block, a page that is not there
      const unsigned vis = (unsigned)seen_keys<TK>(h, s, pages, k0);
      if (vis == 0) return 0;
      const Args a = arguments();
      global_ptr row = !((vis >> l16) & 1) ? dummy : page + l16 * D;
      if (((vis >> l16) & 1) != 0 && k0 + l16 >= s.n)
        row = rows_at(a->kb, 4 * (cur.b * a->kb_st[0] + cur.kvh * a->kb_st[1] + (k0 + l16 - s.n) * a->kb_st[2]));
#pragma unroll
      for (int c = 0; c < NC; ++c) k[c] = *(vec_ptr)(row + 16 * c + 4 * G);
      return vis;
    };
    auto load_v = [&](int k0, unsigned vis) {
      const global_ptr page = rows_at(h.vp, row_offset(h, pages.of(h, k0), cur.kvh, k0, 4 * D));
      if (vis == 0xffffu && k0 + TK <= s.n) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < NV; ++c) v[r][c] = *(vec_ptr)(page + (4 * G + r) * D + 64 * c + 4 * l16);
        return;
      }
      const Args a = arguments();
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 4 * G + r;
        const bool there = (vis >> j) & 1;
        global_ptr row = there ? page + j * D : dummy;
        if (there && k0 + j >= s.n) row = rows_at(a->vb, 4 * (cur.b * a->vb_st[0] + cur.kvh * a->vb_st[1] + (k0 + j - s.n) * a->vb_st[2]));
#pragma unroll
        for (int c = 0; c < NV; ++c) {
          const f32x4 x = *(vec_ptr)(row + 64 * c + 4 * l16);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[r][c][e] = there ? x[e] : 0.f;
        }
      }
    };
    bool taken = false;
    int i = begin;
    unsigned vis_next = load_k(i);
    for (; i < cur.T && left > 0; ++i, --left) {
      const unsigned vis = vis_next;
      const int k0 = s.tile(i) * TK;
      // the values travel under the products of the keys, the next tile's keys under the softmax and the products of the values
      if (vis != 0) load_v(k0, vis);
      // ---- S^T = K Q^T, from 0 in every tile, so that equal keys have equal scores
      f32x4 z[1] = {{0.f, 0.f, 0.f, 0.f}};
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][e], q[c][e], z[0], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      vis_next = i + 1 < cur.T && left > 1 ? load_k(i + 1) : 0;
      __builtin_amdgcn_sched_barrier(0);
      if (vis == 0) continue;
      const bool missing = vis != 0xffffu, above = k0 + TK > all_hi, below = k0 < all_lo && k0 + TK > h.sinks;
      if (missing || above || below) {
        hide<1>(z, k0, lo, hi, h.sinks, vis, missing, above, below);
        if (s.p1 > s.p0) {                         // rows at different positions: what a row does not see must not reach it
          bool bad = false;
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) bad |= !__builtin_isfinite(v[r][c][e]);
          if (__builtin_expect(__ballot(bad) != 0, 0)) {
            taken = true;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[r][c][e] = __builtin_isfinite(v[r][c][e]) ? v[r][c][e] : 0.f;
          }
        }
      }
      float mx = fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3]));
      if (__builtin_amdgcn_ballot_w64(mx > limit) != 0) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float to = mx > limit ? mx : m, corr = exp2_fast((m - to) * h.scale_log2);
        lsum *= corr;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
          for (int b = 0; b < 4; ++b) o[c][b] *= corr;
        m = to;
        limit = m == kNegBig ? kNegBig : m + h.thr8;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[0][e] = exp2_fast((z[0][e] - m) * h.scale_log2);
        lsum += z[0][e];                           // per-lane part, added up over the lanes of a row at the end
      }
      // ---- O^T += V^T P^T
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
          for (int b = 0; b < 4; ++b) o[c][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][c][b], z[0][r], o[c][b], 0, 0, 0);
    }

    // ---- this wave's share of the unit is done: lane (row l16, G) holds columns 64 c + 16 G + 4 r + b
    {
      const Args a = arguments();
      lsum += __shfl_xor(lsum, 16);
      lsum += __shfl_xor(lsum, 32);
      const bool whole = begin == 0 && i == cur.T;
      const int g = a->g, R = row0 + l16;
      const long long slot0 = ((long long)worker * 2 + part) * 16 - row0;
      float* const part_o = TOGETHER ? part_s + (wave * 16LL - row0) * D : a->ws_o + slot0 * D;
      float* const part_ml = TOGETHER ? part_s + NW * 16 * D + 2 * (wave * 16LL - row0) : a->ws_ml + 2 * slot0;
      if (R < cur.s.q_len * g) {
        const float inv = !whole ? 1.f : lsum == 0.f ? 0.f : 1.0f / lsum;
        const int r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
        float* to = whole ? (float*)a->out + cur.b * a->o_st[0] + hq * a->o_st[1] + r * a->o_st[2] : part_o + (long long)R * D;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<f32x4*>(to + 64 * c + 16 * G + 4 * e) = f32x4{o[c][0][e], o[c][1][e], o[c][2][e], o[c][3][e]} * inv;
        if (!whole && G == 0) { part_ml[2 * R] = m; part_ml[2 * R + 1] = lsum; }
      }
      if (taken) put_back<float, D, TK>(cur.s, cur.b, cur.kvh, begin, i, row0, 16, whole, part_o);
      if constexpr (TOGETHER) {
        if (waves > 1) {
          __syncthreads();
          merge_waves<float, D, 64 * NW>(cur, row0, 16, waves, part_s, 16 * D, part_s + NW * 16 * D, 32);
        }
        return;
      }
    }
    part = 1;
    if (left > 0) {
      const int b = cur.b;
      cur.i = cur.T - 1;
      next_tile<TK>(cur);
      if (cur.b != b) pages.open(cur.b);
    }
  }
}

// Waves of a workgroup together, or each for itself (us, together / for itself; heads of 64, 16 and 4 of them, 5 query rows each):
//   fewer units than CUs: few keys: 4 sequences of 600 13 / 16, of 2000 31 / 17 (128 wide, half of that: 1 of 500 18 / 17)
//   else many keys: 32 sequences of 1000 25 / 34, 1024 of 50 to 1000 (4 rows) 221 / 265; 32 and 8 heads of 128, one row: 512 of 50 to
//     200 157 / 115
static bool together(const sdllm_paged_attn_params& p, bool with_block, int row_tiles) {
  const long long tiles = paged_most_tiles(p, with_block, 16, 16);
  const long long units = (long long)p.B * p.Hkv * row_tiles;
  return p.kv_splits == 0 && (units < kNumCUs ? tiles * p.D <= 2560 : tiles >= 32 && units < (1 << 22));   // a launch has fewer than 2^32 threads
}

static int row_tiles_of(const sdllm_paged_attn_params& p) { return (int)(((long long)p.Hq / p.Hkv * p.K + 15) / 16); }

static SharePlan plan_f32(const sdllm_paged_attn_params& p, bool with_block) {
  const int row_tiles = row_tiles_of(p);
  if (together(p, with_block, row_tiles)) return SharePlan{p.B * p.Hkv * row_tiles, 0};
  // Heads of 64 (half the work and the bytes of a tile): two waves to a SIMD and four tiles a share, else one and two.  (us, one and two to
  // a SIMD: 4 sequences of 20000 keys, 16 / 4 heads of 64, 5 rows 68 / 60; 16 of 4096, 32 / 8 heads of 128, 1 row 102 / 107, 1 of 1000 14 / 18.)
  return p.D == 64 ? plan_shares(p, with_block, 16, row_tiles, 16, 8 * kNumCUs, 4) : plan_shares(p, with_block, 16, row_tiles, 16, 4 * kNumCUs, 2);
}

size_t paged_f32_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  return share_bytes(plan_f32(p, with_block), 16, p.D);
}

template <int D>
static hipError_t launch_f32(const PagedArgs& a, bool one_unit, hipStream_t stream, bool launch = true) {
  constexpr size_t together_bytes = 8 * 16 * (D + 2) * sizeof(float);
  static LdsOptIn st;
  if (one_unit) {
    hipError_t e = ensure_lds_opt_in(reinterpret_cast<const void*>(&paged_f32_kernel<D, true>), together_bytes, st);
    if (e != hipSuccess || !launch) return e;
    hipLaunchKernelGGL((paged_f32_kernel<D, true>), dim3(a.workers), dim3(512), together_bytes, stream, a);
  } else {
    hipLaunchKernelGGL((paged_f32_kernel<D, false>), dim3((a.workers + 3) / 4), dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_paged_f32(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream) {
  const int row_tiles = row_tiles_of(p);
  const bool one_unit = together(p, a.kb != nullptr, row_tiles);
  set_shares(a, plan_f32(p, a.kb != nullptr), 16, row_tiles, p.D, workspace);
  hipError_t e = p.D == 128 ? launch_f32<128>(a, one_unit, stream) : launch_f32<64>(a, one_unit, stream);
  if (e != hipSuccess || a.min_tiles == 0) return e;
  return launch_shares_merge(a, p.dtype, p.D, 16, stream);
}

hipError_t prepare_paged_f32() {
  hipError_t e = launch_f32<128>(PagedArgs{}, true, nullptr, false);
  return e == hipSuccess ? launch_f32<64>(PagedArgs{}, true, nullptr, false) : e;
}

}  // namespace sdllm
