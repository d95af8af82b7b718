// fp32 attention over a paged K/V cache (sdllm_paged_attention) on the matrix cores (v_mfma_f32_16x16x4_f32).
//
// A unit is 16 query rows of a (sequence, K/V head).  Every wave walks a contiguous share of all units' 16-key tiles, laid end to end
// as in the bf16 stream kernel; K and V go from memory straight into registers in operand layout, without LDS or barriers.  The
// contraction index and the output column of a matrix instruction may be numbered at will as long as both sides agree:
//   S^T = K Q^T: step (c, e) multiplies d = 16 c + 4 G + e, so that a lane loads 16 bytes of a row of K (and of Q) at a time;
//   O^T = V^T P^T: step r multiplies keys 4 G + r, where the accumulators of S^T already hold P; row i of output block (c, b) is
//         column d = 64 c + 4 i + b, so that 16 bytes of V serve four blocks and a lane ends up with 16 columns in a row.
// Sums, weights and products stay in fp32 throughout.  Few rows and short spans are latency, not bandwidth: 4 sequences, 16 and 4 heads
// of 64, 5 query rows with a window of 1024 and 4 sinks (6.9 MB of K/V), take 14 us here and 5 us in the merge; a wave per query
// row with scalar products took 320 us.
#include "paged_attention.h"

namespace sdllm {

typedef const f32x4* vec_ptr;

template <int D>
__global__ __launch_bounds__(256, 2) void paged_f32_kernel(PagedArgs) {
  constexpr int TK = 16, NC = D / 16, NV = D / 64;
  const int lane = threadIdx.x & 63, l16 = lane & 15, G = lane >> 4;
  const int worker = blockIdx.x * 4 + uniform(threadIdx.x >> 6);
  Unit cur;
  int left;
  {
    const Args a = arguments();
    if (worker >= a->workers) return;
    if (a->min_tiles == 0) {
      const int e = divide(worker, a->by_Hkv);
      open_unit<TK>(cur, e, worker - e * a->Hkv, 0);
      left = cur.T;
    } else {
      left = open_share<TK>(worker, cur);
    }
  }
  if (left == 0) return;
  const Hot h = hot_arguments();
  Pages pages;
  pages.open(cur.b);
  int part = 0;
  while (left > 0) {
    const int begin = cur.i;
    f32x4 q[NC];
    int lo, hi, all_hi, all_lo, row0;
    const float* dummy;                            // a row that exists, for keys that do not
    {
      const Args a = arguments();
      const int g = a->g, last_row = cur.s.q_len * g - 1;
      row0 = cur.rt * 16;
      const int R = min(row0 + l16, last_row), r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
      const float* qp = (const float*)a->q + cur.b * a->q_st[0] + hq * a->q_st[1] + r * a->q_st[2];
      dummy = qp;
#pragma unroll
      for (int c = 0; c < NC; ++c) q[c] = *(vec_ptr)(qp + 16 * c + 4 * G);
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
    bool redo = false;
    int i = begin;
    for (; i < cur.T && left > 0; ++i, --left) {
      const Seen& s = cur.s;
      if (s.tiles == 0) continue;
      const int k0 = s.tile(i) * TK;
      pages.seek(h, k0);
      const float* kpage = (const float*)(h.kp + row_offset(h, pages.of(h, k0), cur.kvh, k0, 4 * D));
      const float* vpage = (const float*)(h.vp + row_offset(h, pages.of(h, k0), cur.kvh, k0, 4 * D));
      f32x4 k[NC], v[4][NV];
      unsigned vis = 0xffffu;
      if (pages.ok(h, k0) && ((k0 >= s.lo && k0 <= s.last16) || k0 <= s.sink16)) {
#pragma unroll
        for (int c = 0; c < NC; ++c) k[c] = *(vec_ptr)(kpage + l16 * D + 16 * c + 4 * G);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < NV; ++c) v[r][c] = *(vec_ptr)(vpage + (4 * G + r) * D + 64 * c + 4 * l16);
      } else {
        // a border of what is seen, the end of the cache, rows of the block, a page that is not there
        vis = (unsigned)seen_keys<TK>(h, s, pages, k0);
        if (vis == 0) continue;
        const Args a = arguments();
        const float *kb = nullptr, *vb = nullptr;
        if (a->kb != nullptr) {
          kb = (const float*)a->kb + cur.b * a->kb_st[0] + cur.kvh * a->kb_st[1] + (k0 - s.n) * a->kb_st[2];
          vb = (const float*)a->vb + cur.b * a->vb_st[0] + cur.kvh * a->vb_st[1] + (k0 - s.n) * a->vb_st[2];
        }
        const float* kr = !((vis >> l16) & 1) ? dummy : k0 + l16 < s.n ? kpage + l16 * D : kb + l16 * a->kb_st[2];
#pragma unroll
        for (int c = 0; c < NC; ++c) k[c] = *(vec_ptr)(kr + 16 * c + 4 * G);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = 4 * G + r;
          const bool there = (vis >> j) & 1;
          const float* vr = !there ? dummy : k0 + j < s.n ? vpage + j * D : vb + j * a->vb_st[2];
#pragma unroll
          for (int c = 0; c < NV; ++c) {
            const f32x4 x = *(vec_ptr)(vr + 64 * c + 4 * l16);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[r][c][e] = there ? x[e] : 0.f;
          }
        }
      }
      // ---- S^T = K Q^T, from 0 in every tile, so that equal keys have equal scores
      f32x4 z[1] = {{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][e], q[c][e], z[0], 0, 0, 0);
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
            redo = true;
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
      if (R < cur.s.q_len * g) {
        const float inv = !whole ? 1.f : lsum == 0.f ? 0.f : 1.0f / lsum;
        const int r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
        float* to = whole ? (float*)a->out + cur.b * a->o_st[0] + hq * a->o_st[1] + r * a->o_st[2] : a->ws_o + (slot0 + R) * D;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<f32x4*>(to + 64 * c + 16 * G + 4 * e) = f32x4{o[c][0][e], o[c][1][e], o[c][2][e], o[c][3][e]} * inv;
        if (!whole && G == 0) { a->ws_ml[2 * (slot0 + R)] = m; a->ws_ml[2 * (slot0 + R) + 1] = lsum; }
      }
      if (redo) redo_rows<float, D, TK>(cur.s, cur.b, cur.kvh, begin, i, row0, 16, whole, slot0);
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

static SharePlan plan_f32(const sdllm_paged_attn_params& p, bool with_block) {
  const int row_tiles = (int)(((long long)p.Hq / p.Hkv * p.K + 15) / 16);
  return plan_shares(p, with_block, 16, row_tiles, 16, 8 * kNumCUs, 4);
}

size_t paged_f32_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  return share_bytes(plan_f32(p, with_block), 16, p.D);
}

hipError_t launch_paged_f32(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream) {
  set_shares(a, plan_f32(p, a.kb != nullptr), 16, (a.R + 15) / 16, p.D, workspace);
  const dim3 grid((a.workers + 3) / 4);
  if (p.D == 128) hipLaunchKernelGGL(paged_f32_kernel<128>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(paged_f32_kernel<64>, grid, dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.min_tiles == 0) return e;
  return launch_shares_merge(a, p.dtype, p.D, 16, stream);
}

}  // namespace sdllm
