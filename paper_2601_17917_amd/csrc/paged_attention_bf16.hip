// bf16 attention over a paged K/V cache for gfx950 (sdllm_paged_attention), few query rows per (sequence, K/V head): one token, a
// few tokens, a block of up to 32 rows over its heads.
//
// Bound by the read of K and V.  Every wave is a stream of its own: it walks a contiguous range of key tiles of the whole call
// -- sequences, their K/V heads, their tiles, laid end to end -- so that all waves carry the same number of tiles whatever the
// lengths are, and meets no other wave.  A tile (8 KiB of K and 8 KiB of V) goes global -> LDS into the wave's own 16 KiB, from
// there into registers in operand layout, and the next tile's transfers go in flight into the same 16 KiB while the products and
// the softmax of this one run.
//   S^T = K Q^T, O^T = V^T P^T with v_mfma_f32_16x16x32_bf16, operands laid out as in the dense kernel (rows padded to 16 or 32).
//   Online softmax: the product's accumulators start at minus the row's reference, so that it yields s - reference and a weight is
//   one multiply and one exponential, whatever the scores' size; the reference moves only where a maximum exceeds it by 8 in log2
//   units.  The second product takes bf16, and a weight goes in as two: the next number below it, and what is missing, rounded (2^-15 of the
//   weight is lost at most).  Neither is negative or, down to weights of 2^-100, zero: infinite values keep their sign.  K and V are read at
//   HBM's rate, which leaves the matrix unit the room: as one number each, which loses 2^-8, a token over 700 keys takes 7.1 us instead of 7.3,
//   over 32 sequences of 8192 168.0 instead of 168.4, 32 rows of 8 sequences of 2000 keys (8 heads of 64) 17.9 instead of 18.9.  The row sums
//   are those of the same numbers; all sums are fp32.
// A (sequence, head) that one wave walked alone is written at once; of the others every wave leaves (O, m, l), merged in tile order
// by a second launch.  Which wave does what follows from the lengths alone: no atomics, the same result every time.
//   TOGETHER: the eight waves of a workgroup share the tiles of one (sequence, K/V head) and merge through LDS: no second launch.
// Measured, one row over 32 and 8 heads of 128: 32 sequences of 200 to 16384 keys, 501 MB, 80 + 5 us (5.9 TB/s); 64 of 4096, 1.07 GB,
// 168 us (6.4 TB/s); one of 700, 7.3 us; one of 32768, 134 MB, 31 us.
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

template <int D, int RB, bool TOGETHER>
__global__ __launch_bounds__(TOGETHER ? 512 : 256, 2) void paged_stream_kernel(PagedArgs) {
  using S = StreamShape<D>;
  constexpr int TK = S::TK, KB = S::KB, NS = S::NS, NDB = S::NDB, U = TK / 32;
  constexpr int NW = TOGETHER ? 8 : 4;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63, l16 = lane & 15, G = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  unsigned char* lds_wave = lds + wave * S::WAVEB;

  // this wave's tiles
  const int worker = TOGETHER ? blockIdx.x : blockIdx.x * NW + wave;
  const Hot h = hot_arguments();
  Pages pages;
  Unit nxt;
  int left;                                        // tiles of its share still to do
  {
    const Args a = arguments();
    if (worker >= a->workers) return;
    if (a->min_tiles == 0) {                       // a wave, or a workgroup, per (sequence, K/V head)
      open_whole_unit<TK>(nxt, pages, h, worker);
      left = nxt.T;
    } else {
      left = open_share<TK>(worker, nxt);
      pages.open(nxt.b);
    }
  }
  [[maybe_unused]] int waves = 0;                  // of the workgroup that have tiles
  if constexpr (TOGETHER) {
    const int per = (left + NW - 1) / NW;
    if (left == 0) return;
    waves = (left + per - 1) / per;
    nxt.i = wave * per;
    left = min(per, left - nxt.i);
    if (left <= 0) {
      if (waves > 1) {                             // the barrier that the waves with tiles come to
        __syncthreads();
        merge_waves<uint16_t, D, 64 * NW>(nxt, 0, 16 * RB, waves, (const float*)lds, S::WAVEB / 4, (const float*)(lds + NW * S::WAVEB), 32 * RB);
      }
      return;
    }
  }
  if (left == 0) return;
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
        const int R = min(16 * rb + l16, last_row), r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
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
    bool taken = false;
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
        if (!TOGETHER && nxt.b != cur.b) pages.open(nxt.b);
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
      s16x8 pk[RB][U], rest[RB][U];                // the next bf16 number below, and what is missing: both positive
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
          union { uint32_t w[4]; s16x8 v; } p, q;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = sacc[rb][2 * u + i / 2][2 * (i % 2)], y = sacc[rb][2 * u + i / 2][2 * (i % 2) + 1];
            const unsigned x1 = __builtin_elementwise_sub_sat(__float_as_uint(x), 1u), y1 = __builtin_elementwise_sub_sat(__float_as_uint(y), 1u);
            p.w[i] = __builtin_amdgcn_perm(y1, x1, 0x07060302);               // their upper halves
            q.w[i] = pack_bf16x2(x - __uint_as_float(x1 & 0xffff0000u), y - __uint_as_float(y1 & 0xffff0000u));
          }
          pk[rb][u] = p.v; rest[rb][u] = q.v;
        }
        // row sums on the matrix pipe, from what the values are weighted with
        union { uint32_t w[4]; s16x8 v; } ones;
        ones.w[0] = ones.w[1] = ones.w[2] = ones.w[3] = 0x3f803f80u;
        f32x4 ls = {lsum[rb], 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
          ls = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones.v), __builtin_bit_cast(bf16x8, pk[rb][u]), ls, 0, 0, 0);
          ls = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones.v), __builtin_bit_cast(bf16x8, rest[rb][u]), ls, 0, 0, 0);
        }
        lsum[rb] = ls[0];
      }
      if (masked && cur.s.p1 > cur.s.p0) {         // rows at different positions: what a row does not see must not reach it
        unsigned bad = 0;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int db = 0; db < NDB; ++db) bad |= nonfinite_bits(__builtin_bit_cast(u32x4, vop[u][db]));
        if (__builtin_expect(__ballot(bad != 0) != 0, 0)) {
          taken = true;
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
          for (int rb = 0; rb < RB; ++rb) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, vop[u][db]);
            o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, pk[rb][u]), o[rb][db], 0, 0, 0);
            o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, rest[rb][u]), o[rb][db], 0, 0, 0);
          }
    }

    // ---- this wave's share of the unit is done
    const Args a = arguments();
    const bool whole = begin == 0 && i == cur.T;
    const int g = a->g, last_row = cur.s.q_len * g - 1;
    const long long slot0 = ((long long)worker * 2 + part) * a->R;
    float* const part_o = TOGETHER ? (float*)lds_wave : a->ws_o + slot0 * D;
    float* const part_ml = TOGETHER ? (float*)(lds + NW * S::WAVEB) + wave * 32 * RB : a->ws_ml + 2 * slot0;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int R = 16 * rb + l16;
      if (R > last_row) continue;
      if (whole) {
        const float inv = lsum[rb] == 0.f ? 0.f : 1.0f / lsum[rb];
        const int r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
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
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4*>(part_o + R * D + 16 * db + 4 * G) = o[rb][db];
        if (G == 0) { part_ml[2 * R] = thr[rb] == kNegBig ? kNegBig : -neg_m[rb][0]; part_ml[2 * R + 1] = lsum[rb]; }
      }
    }
    if (taken) put_back<uint16_t, D, TK>(cur.s, cur.b, cur.kvh, begin, i, 0, 16 * RB, whole, part_o);
    if constexpr (TOGETHER) {
      if (waves > 1) {
        __syncthreads();
        merge_waves<uint16_t, D, 64 * NW>(cur, 0, 16 * RB, waves, (const float*)lds, S::WAVEB / 4, (const float*)(lds + NW * S::WAVEB), 32 * RB);
      }
      return;
    }
    part = 1;
  }
}

// Waves that share the tiles: one to a SIMD.  Two fit, but do not read faster, and leave twice as much to merge (us, one and two: 1 sequence
// of 16384 keys, 32 / 8 heads of 128, 21 / 23; 32 sequences of 8192 168 / 168; 28 / 4 heads, 4 rows, 32 sequences of 8000 96 / 105).
// A share has two tiles at least: of one, 1 sequence of 2048 keys 11.6 against 12.1, of 4096 13.8 against 13.2; of three 14.1, 14.8.
static constexpr int kStreamWaves = 4 * kNumCUs;
static constexpr int kStreamMinTiles = 2;
// Waves of a workgroup together, or each for itself (us, 32 query and 8 K/V heads of 128, one row each; together / for itself):
//   up to 4 units per CU: few keys, where a second launch for the merge costs more than idle CUs do, or no fewer workgroups busy:
//     1 sequence of 128 keys 5.2 / 10.3, of 1024 11.7 / 11.9, of 2048 21 / 12; 32 of 1024 24 / 30
//   more: many keys, where a workgroup's start is a small part of its time: 128 sequences of 100 to 4000 keys 185 / 194, 512 of 50 to
//     1000 182 / 195, 512 of 50 to 200 85 / 48
static bool together(const sdllm_paged_attn_params& p, bool with_block) {
  const long long tiles = paged_most_tiles(p, with_block, (long long)p.Hq / p.Hkv * p.K, 4096 / p.D);
  return p.kv_splits == 0 && ((long long)p.B * p.Hkv < 4 * kNumCUs ? tiles <= 32 : tiles >= 24);
}

static SharePlan plan_stream(const sdllm_paged_attn_params& p, bool with_block) {
  if (together(p, with_block)) return SharePlan{p.B * p.Hkv, 0};
  return plan_shares(p, with_block, p.Hq / p.Hkv * p.K, 1, 4096 / p.D, kStreamWaves, kStreamMinTiles);
}

size_t paged_stream_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  return share_bytes(plan_stream(p, with_block), p.Hq / p.Hkv * p.K, p.D);
}

template <int D, int RB>
static hipError_t launch_stream(const PagedArgs& a, bool one_unit, hipStream_t stream, bool launch = true) {
  constexpr int wave_bytes = StreamShape<D>::WAVEB, together_bytes = 8 * (wave_bytes + 128 * RB);
  static LdsOptIn st;
  if (one_unit) {
    hipError_t e = ensure_lds_opt_in(reinterpret_cast<const void*>(&paged_stream_kernel<D, RB, true>), together_bytes, st);
    if (e != hipSuccess || !launch) return e;
    hipLaunchKernelGGL((paged_stream_kernel<D, RB, true>), dim3(a.workers), dim3(512), together_bytes, stream, a);
  } else {
    hipLaunchKernelGGL((paged_stream_kernel<D, RB, false>), dim3((a.workers + 3) / 4), dim3(256), 4 * wave_bytes, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_paged_stream(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream) {
  const bool one_unit = together(p, a.kb != nullptr);
  set_shares(a, plan_stream(p, a.kb != nullptr), a.R, 1, p.D, workspace);
  hipError_t e;
  if (p.D == 128) e = a.R <= 16 ? launch_stream<128, 1>(a, one_unit, stream) : launch_stream<128, 2>(a, one_unit, stream);
  else e = a.R <= 16 ? launch_stream<64, 1>(a, one_unit, stream) : launch_stream<64, 2>(a, one_unit, stream);
  if (e != hipSuccess || a.min_tiles == 0) return e;
  return launch_shares_merge(a, p.dtype, p.D, 4096 / p.D, stream);
}

hipError_t prepare_paged_stream() {
  hipError_t e = launch_stream<128, 1>(PagedArgs{}, true, nullptr, false);
  if (e == hipSuccess) e = launch_stream<128, 2>(PagedArgs{}, true, nullptr, false);
  if (e == hipSuccess) e = launch_stream<64, 1>(PagedArgs{}, true, nullptr, false);
  if (e == hipSuccess) e = launch_stream<64, 2>(PagedArgs{}, true, nullptr, false);
  return e;
}

}  // namespace sdllm
