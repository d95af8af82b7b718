// bf16 attention over a paged K/V cache for gfx950 (sdllm_paged_attention), few query rows per (sequence, K/V head): one token, a
// few tokens, a block of up to 32 rows over its heads.
//
// Bound by the read of K and V.  Every wave is a stream of its own: it walks a contiguous range of key tiles of the whole call
// -- sequences, their K/V heads, their tiles, laid end to end -- so that all waves carry the same number of tiles whatever the
// lengths are, and meets no other wave.  A tile (8 KiB of K and 8 KiB of V) goes global -> LDS into the wave's own 16 KiB, from
// there into registers in operand layout, and the next tile's transfers go in flight into the same 16 KiB while the products and
// the softmax of this one run: with eight waves on a CU some 100 KiB are in flight all the time.
//   S^T = K Q^T, O^T = V^T P^T with v_mfma_f32_16x16x32_bf16, operands laid out as in the dense kernel (rows padded to 16 or 32).
//   Online softmax: the product's accumulators start at minus the row's reference, so that it yields s - reference and a weight is
//   one multiply and one exponential, whatever the scores' size; the reference moves only where a maximum exceeds it by 8 in log2
//   units.
// A (sequence, head) that one wave walked alone is written at once; of the others every wave leaves (O, m, l), merged in tile order
// by a second launch.  Which wave does what follows from the lengths alone: no atomics, the same result every time.
#include "paged_attention.h"

namespace sdllm {

template <int D> struct StreamShape {
  static constexpr int TK = 4096 / D;              // keys per tile
  static constexpr int KB = TK / 16;               // 16-key slabs
  static constexpr int NS = D / 32, NDB = D / 16, ROWB = D * 2;
  static constexpr int SLABB = 16 * ROWB, VB = TK * ROWB, WAVEB = 2 * VB;
};

// Puts tile u.i in flight.  Returns which of its keys some query row sees (bit r: key r; the rows of the others are zero).
template <int D>
__device__ __forceinline__ unsigned long long issue_tile(const Hot& h, const Unit& u, Pages& pages, unsigned base,
                                                         unsigned char* lds_wave) {
  using S = StreamShape<D>;
  const Seen& s = u.s;
  if (s.tiles == 0) return 0;                      // nothing to see, nothing is read from LDS either
  const int k0 = s.tile(u.i) * S::TK;
  pages.seek(h, k0);
  constexpr unsigned long long kAll = S::TK == 64 ? ~0ull : (1ull << S::TK) - 1;
  const bool plain = pages.all_ok<S::TK>(h, k0) && ((k0 >= s.lo && k0 + S::TK - 16 <= s.last16) || k0 + S::TK - 16 <= s.sink16);
  const unsigned long long vis = plain ? kAll : seen_keys<S::TK>(h, s, pages, k0);
#pragma unroll
  for (int j = 0; j < S::KB; ++j) {
    const int k = k0 + 16 * j;
    const unsigned bits = (unsigned)(vis >> (16 * j)) & 0xffffu;
    const unsigned long long at = row_offset(h, pages.of(h, k), u.kvh, k, S::ROWB);
    if (bits == 0xffffu && k + 16 <= s.n) {
      move_slab<D, true, false>(base + j * S::SLABB, h.kp + at);
      move_slab<D, true, true>(base + S::VB + j * S::SLABB, h.vp + at);
    } else {
      move_rows<D, true, false>(s, u.b, u.kvh, k, bits, h.kp + at, base + j * S::SLABB, lds_wave + j * S::SLABB);
      move_rows<D, true, true>(s, u.b, u.kvh, k, bits, h.vp + at, base + S::VB + j * S::SLABB, lds_wave + S::VB + j * S::SLABB);
    }
  }
  return vis;
}

template <int D, int RB>
__global__ __launch_bounds__(256, 2) void paged_stream_kernel(PagedArgs) {
  using S = StreamShape<D>;
  constexpr int TK = S::TK, KB = S::KB, NS = S::NS, NDB = S::NDB, U = TK / 32;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * S::WAVEB];
  const int lane = threadIdx.x & 63, l16 = lane & 15, G = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  unsigned char* lds_wave = lds + wave * S::WAVEB;

  // this wave's tiles
  const int worker = blockIdx.x * 4 + wave;
  Unit nxt;
  int left;                                        // tiles of its share still to do
  {
    const Args a = arguments();
    if (worker >= a->workers) return;
    if (a->min_tiles == 0) {                       // a wave per (sequence, K/V head)
      open_unit<TK>(nxt, worker / a->Hkv, worker % a->Hkv, 0);
      left = nxt.T;
    } else {
      left = open_share<TK>(worker, nxt);
    }
  }
  if (left == 0) return;
  const Hot h = hot_arguments();
  Pages pages;
  pages.open(nxt.b);
  const unsigned base = uniform((int)(unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)lds_wave);
  unsigned long long vis_next = issue_tile<D>(h, nxt, pages, base, lds_wave);
  // LDS offsets of the lane's operands of slice 0 / d block 0; the others flip bits of them
  const unsigned kro = l16 * S::ROWB + ((G ^ ((D == 128) ? l16 : (l16 >> 1))) << 4);
  const int e4 = l16 >> 2, c4 = l16 & 3, fv = (D == 128) ? 2 * (4 * (G & 1) + e4) : 2 * (2 * (G & 1) + (e4 >> 1));
  const unsigned vro = S::VB + (4 * G + e4) * S::ROWB + (((c4 >> 1) ^ fv) << 4) + ((c4 & 1) << 3);

  int part = 0;                                    // of this wave: the first unit's partial result goes to slot 0, the last's to 1
  while (left > 0) {
    // ---- a unit: its query rows as MFMA B operands (lane: row l16, d = 32 s + 8 G .. + 7)
    const Unit cur = nxt;
    const int begin = cur.i;
    bf16x8 qreg[RB][NS];
    int lo[RB], hi[RB], all_hi, all_lo;            // keys that row l16 sees, that all rows see
    {
      const Args a = arguments();
      const int g = a->g, last_row = cur.s.q_len * g - 1;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int R = min(16 * rb + l16, last_row), r = R / g, hq = cur.kvh * g + R - r * g;
        const uint16_t* qp = (const uint16_t*)a->q + cur.b * a->q_st[0] + hq * a->q_st[1] + r * a->q_st[2];
#pragma unroll
        for (int s2 = 0; s2 < NS; ++s2) qreg[rb][s2] = *reinterpret_cast<const bf16x8*>(qp + 32 * s2 + 8 * G);
        row_range(a, cur.s, r, lo[rb], hi[rb]);
      }
      int x;
      row_range(a, cur.s, 0, x, all_hi);
      row_range(a, cur.s, max(cur.s.q_len - 1, 0), all_lo, x);
    }
    f32x4 o[RB][NDB];
    f32x4 neg_m[RB];                               // minus the reference of row l16, in score units, four times
    float thr[RB], lsum[RB];                       // kNegBig: no reference yet
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      neg_m[rb] = f32x4{0.f, 0.f, 0.f, 0.f}; thr[rb] = kNegBig; lsum[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    bool redo = false;
    int i = begin;
    for (; i < cur.T && left > 0; ++i, --left) {
      const unsigned long long vis = vis_next;
      wait_transfers();
      bf16x8 kop[KB][NS];
      s16x8 vop[U][NDB];
      if (cur.s.tiles > 0) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int s2 = 0; s2 < NS; ++s2) kop[kb][s2] = *reinterpret_cast<const bf16x8*>(lds_wave + (kro ^ (s2 << 6)) + kb * S::SLABB);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(lds_wave + (vro ^ (db << 5)) + 32 * u * S::ROWB));
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(lds_wave + (vro ^ (db << 5)) + (32 * u + 16) * S::ROWB));
            vop[u][db] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
          }
      }
      // the operands are in registers: the area takes the next tile
      wait_lds();
      if (left > 1) {
        next_tile<TK>(nxt);
        if (nxt.b != cur.b) pages.open(nxt.b);
        vis_next = issue_tile<D>(h, nxt, pages, base, lds_wave);
      }
      if (vis == 0) continue;

      // ---- S^T = K Q^T
      f32x4 sacc[RB][KB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) sacc[rb][kb] = neg_m[rb];
#pragma unroll
      for (int s2 = 0; s2 < NS; ++s2)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            sacc[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[kb][s2], qreg[rb][s2], sacc[rb][kb], 0, 0, 0);
      const int k0 = cur.s.tile(i) * TK;
      constexpr unsigned long long kAll = KB == 4 ? ~0ull : (1ull << (16 * KB)) - 1;
      const bool missing = vis != kAll, above = k0 + TK > all_hi, below = k0 < all_lo && k0 + TK > h.sinks;
      const bool masked = missing || above || below;
      if (masked) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) hide<KB>(sacc[rb], k0, lo[rb], hi[rb], h.sinks, vis, missing, above, below);
      }
      // ---- online softmax: p = exp2((s - reference) scale_log2)
      s16x8 pk[RB][U];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          mx = fmaxf(fmaxf(fmaxf(mx, sacc[rb][kb][0]), fmaxf(sacc[rb][kb][1], sacc[rb][kb][2])), sacc[rb][kb][3]);
        if (__builtin_amdgcn_ballot_w64(mx > thr[rb]) != 0) {
          const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
          mx = fmaxf(__uint_as_float(s16[0]), __uint_as_float(s16[1]));
          const auto s32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
          mx = fmaxf(__uint_as_float(s32[0]), __uint_as_float(s32[1]));
          const bool move = mx > thr[rb];
          const float shift = move ? mx : 0.f;
          const float corr = thr[rb] == kNegBig ? 0.f : exp2_fast(-shift * h.scale_log2);
          lsum[rb] *= corr;
#pragma unroll
          for (int db = 0; db < NDB; ++db) o[rb][db] *= corr;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) sacc[rb][kb] -= shift;
          neg_m[rb] -= shift;
          thr[rb] = move ? h.thr8 : thr[rb];
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) sacc[rb][kb][e] = exp2_fast(sacc[rb][kb][e] * h.scale_log2);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          union { uint32_t w[4]; s16x8 v; } cv;
          cv.w[0] = pack_bf16x2(sacc[rb][2 * u][0], sacc[rb][2 * u][1]);
          cv.w[1] = pack_bf16x2(sacc[rb][2 * u][2], sacc[rb][2 * u][3]);
          cv.w[2] = pack_bf16x2(sacc[rb][2 * u + 1][0], sacc[rb][2 * u + 1][1]);
          cv.w[3] = pack_bf16x2(sacc[rb][2 * u + 1][2], sacc[rb][2 * u + 1][3]);
          pk[rb][u] = cv.v;
        }
        // row sums on the matrix pipe, from the rounded probabilities that the values are weighted with
        union { uint32_t w[4]; s16x8 v; } ones;
        ones.w[0] = ones.w[1] = ones.w[2] = ones.w[3] = 0x3f803f80u;
        f32x4 ls = {lsum[rb], 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
          ls = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones.v), __builtin_bit_cast(bf16x8, pk[rb][u]), ls, 0, 0, 0);
        lsum[rb] = ls[0];
      }
      if (masked && cur.s.p1 > cur.s.p0) {         // rows at different positions: what a row does not see must not reach it
        unsigned bad = 0;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int db = 0; db < NDB; ++db) bad |= nonfinite_bits(__builtin_bit_cast(u32x4, vop[u][db]));
        if (__builtin_expect(__ballot(bad != 0) != 0, 0)) {
          redo = true;
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int db = 0; db < NDB; ++db) vop[u][db] = finite_part(vop[u][db]);
        }
      }
      // ---- O^T += V^T P^T
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vop[u][db]),
                                                                __builtin_bit_cast(bf16x8, pk[rb][u]), o[rb][db], 0, 0, 0);
    }

    // ---- this wave's share of the unit is done
    const Args a = arguments();
    const bool whole = begin == 0 && i == cur.T;
    const int g = a->g, last_row = cur.s.q_len * g - 1;
    const long long slot0 = ((long long)worker * 2 + part) * a->R;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int R = 16 * rb + l16;
      if (R > last_row) continue;
      if (whole) {
        const float inv = lsum[rb] == 0.f ? 0.f : 1.0f / lsum[rb];
        const int r = R / g, hq = cur.kvh * g + R - r * g;
        uint16_t* orow = (uint16_t*)a->out + cur.b * a->o_st[0] + hq * a->o_st[1] + r * a->o_st[2];
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          uint2 w;
          w.x = pack_bf16x2(o[rb][db][0] * inv, o[rb][db][1] * inv);
          w.y = pack_bf16x2(o[rb][db][2] * inv, o[rb][db][3] * inv);
          *reinterpret_cast<uint2*>(orow + 16 * db + 4 * G) = w;
        }
      } else {
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4*>(a->ws_o + (slot0 + R) * D + 16 * db + 4 * G) = o[rb][db];
        if (G == 0) { a->ws_ml[2 * (slot0 + R)] = thr[rb] == kNegBig ? kNegBig : -neg_m[rb][0]; a->ws_ml[2 * (slot0 + R) + 1] = lsum[rb]; }
      }
    }
    if (redo) redo_rows<D, TK>(cur.s, cur.b, cur.kvh, begin, i, 0, 16 * RB, whole, slot0);
    part = 1;
  }
}

// Merges the shares of every output row that several workers (waves here, workgroups of the tile kernel) walked, in the order of the tiles.  A workgroup per row: 256 / (D / 4)
// groups of lanes take every so many-th share, then one adds up the groups, in order.
template <int D, int TK>
__global__ __launch_bounds__(256) void shares_merge_kernel(PagedArgs) {
  const Args a = arguments();
  constexpr int TPR = D / 4, NG = 256 / TPR;
  __shared__ f32x4 o_s[NG][TPR];
  __shared__ float m_s[NG], l_s[NG];
  const unsigned unit = blockIdx.x / (unsigned)a->R;
  const int R = blockIdx.x - unit * a->R, b = unit / (unsigned)a->Hkv, kvh = unit - b * a->Hkv;
  // where the unit's tiles lie among the call's
  const int lane = threadIdx.x & 63;
  long long total = 0, start = 0;
  int T = 0, q_len = 0;
  for (int b0 = 0; b0 < a->B; b0 += 64) {
    const int t = tiles_of<TK>(a, b0 + lane), upto = wave_scan(t);
    if (b >= b0 && b < b0 + 64) {
      T = uniform(__shfl(t, b - b0));
      start = (total + uniform(__shfl(upto, b - b0)) - T) * a->Hkv + (long long)kvh * T;
    }
    total += uniform(__shfl(upto, 63));
  }
  total *= a->Hkv;
  q_len = min(max(a->q_lens ? a->q_lens[b] : a->K, 0), a->K);
  if (T == 0 || R >= q_len * a->g) return;
  const long long per = tiles_per_worker(a, total);
  const int w0 = (int)(start / per), w1 = (int)((start + T - 1) / per);
  if (w0 == w1) return;                            // written by its wave
  const int grp = threadIdx.x / TPR, d = (threadIdx.x % TPR) * 4;
  float M = kNegBig, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int w = w0 + grp; w <= w1; w += NG) {
    // the unit is its wave's first one unless the wave began before it
    const long long slot = ((long long)w * 2 + (start > w * per ? 1 : 0)) * a->R + R;
    const f32x4 ov = *reinterpret_cast<const f32x4*>(a->ws_o + slot * D + d);
    const float mk = a->ws_ml[2 * slot], lk = a->ws_ml[2 * slot + 1];
    const float up = fmaxf(M, mk), c0 = exp2_fast((M - up) * a->scale_log2), c1 = exp2_fast((mk - up) * a->scale_log2);
    acc = acc * c0 + ov * c1;
    l = l * c0 + lk * c1;
    M = up;
  }
  o_s[grp][threadIdx.x % TPR] = acc;
  if (d == 0) { m_s[grp] = M; l_s[grp] = l; }
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int k = 1; k < NG; ++k) {
    const float up = fmaxf(M, m_s[k]), c0 = exp2_fast((M - up) * a->scale_log2), c1 = exp2_fast((m_s[k] - up) * a->scale_log2);
    acc = acc * c0 + o_s[k][threadIdx.x % TPR] * c1;
    l = l * c0 + l_s[k] * c1;
    M = up;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int r = R / a->g, h = kvh * a->g + R - r * a->g;
  uint2 w2;
  w2.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  w2.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<uint2*>((uint16_t*)a->out + b * a->o_st[0] + h * a->o_st[1] + r * a->o_st[2] + d) = w2;
}

// ---- launch plan, from the parameters alone
constexpr int kStreamWaves = 8 * kNumCUs;          // resident at once: two workgroups of 64 KiB per CU
constexpr int kStreamMinTiles = 2;
constexpr int kStreamMaxRows = 32;

struct StreamPlan { int workers, min_tiles; bool merge; };

static StreamPlan plan_stream(const sdllm_paged_attn_params& p, bool with_block) {
  const long long TK = 4096 / p.D, units = (long long)p.B * p.Hkv;
  const long long N = p.max_kv_len + (with_block ? p.K : 0);
  long long tiles = (N + TK - 1) / TK;             // most a unit can have
  if (p.window > 0) {
    const long long seen = (p.window + p.K + TK - 2) / TK + 1 + (p.sinks + TK - 1) / TK;
    if (seen < tiles) tiles = seen;
  }
  if (tiles < 1) tiles = 1;
  StreamPlan pl;
  long long per = kStreamMinTiles;
  if (p.kv_splits > 0) per = (tiles + p.kv_splits - 1) / p.kv_splits;
  pl.merge = !(p.kv_splits == 1 || units * (p.Hq / p.Hkv) * p.K >= (1 << 24) || (p.kv_splits == 0 && (units >= 2 * kStreamWaves || p.B > 1024 || tiles <= per)));
  if (!pl.merge) {
    pl.workers = (int)units; pl.min_tiles = 0;
    return pl;
  }
  pl.min_tiles = (int)per;
  long long w = (units * tiles + per - 1) / per;
  const long long most = p.kv_splits > 0 ? 1 << 20 : kStreamWaves;
  pl.workers = (int)(w < most ? w : most);
  return pl;
}

size_t paged_stream_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  const StreamPlan pl = plan_stream(p, with_block);
  return pl.merge ? (size_t)pl.workers * 2 * (size_t)(p.Hq / p.Hkv) * p.K * (p.D + 2) * sizeof(float) : 0;
}

hipError_t launch_shares_merge(const PagedArgs& a, int D, int TK, hipStream_t stream) {
  const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.R));
  if (D == 64) hipLaunchKernelGGL((shares_merge_kernel<64, 64>), grid, dim3(256), 0, stream, a);
  else if (TK == 32) hipLaunchKernelGGL((shares_merge_kernel<128, 32>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((shares_merge_kernel<128, 64>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <int D>
static hipError_t launch_stream(const PagedArgs& a, const StreamPlan& pl, hipStream_t stream) {
  const dim3 grid((pl.workers + 3) / 4);
  if (a.R <= 16) hipLaunchKernelGGL((paged_stream_kernel<D, 1>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_stream_kernel<D, 2>), grid, dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !pl.merge) return e;
  return launch_shares_merge(a, D, 4096 / D, stream);
}

hipError_t launch_paged_stream(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream) {
  const StreamPlan pl = plan_stream(p, a.kb != nullptr);
  a.workers = pl.workers; a.min_tiles = pl.min_tiles;
  a.ws_o = (float*)workspace;
  a.ws_ml = a.ws_o ? a.ws_o + (size_t)pl.workers * 2 * a.R * p.D : nullptr;
  return p.D == 128 ? launch_stream<128>(a, pl, stream) : launch_stream<64>(a, pl, stream);
}

}  // namespace sdllm
