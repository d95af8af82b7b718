// bf16 attention over a paged K/V cache for gfx950 (sdllm_paged_attention), more than 32 query rows per (sequence, K/V head): the
// rows of a block over its heads, the pieces of prompts.
//
// A workgroup owns 16 RB NW query rows (NW waves, 16 RB rows each) and walks key tiles of 64 that its waves share through a
// two-stage ring in LDS: each wave moves 16-row slabs global -> LDS, one tile ahead of the one being computed, one barrier per
// tile.  Products, operand layouts and the softmax are those of the stream kernel.
//   FLAT: one row tile covers a (sequence, K/V head).  The workgroups walk equal shares of all key tiles of the call, laid end to end
//         as the stream kernel's waves do, so that lengths need not be alike.
//   else: a workgroup per (row tile, sequence, K/V head, part of the keys it sees); the tiles of the last rows, which see most under a
//         causal mask, come first.
#include "paged_attention.h"

namespace sdllm {

constexpr int kTK = 64;                            // keys per tile

template <int D, int NST> struct TileShape {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, IPT = 16 / RPI, R256 = 16 / CPR;
  static constexpr int NS = D / 32, NDB = D / 16, ROWB = D * 2;
  static constexpr int SLABB = 16 * ROWB, STAGEB = kTK * ROWB, VB = NST * STAGEB, LDS = 2 * NST * STAGEB + NST * 16;
};

// Moves the 16-row slab `slab` of the tile at key k0 into LDS: K (kind 0), V (kind 1) or both.  Returns which of its rows hold a key that
// some query row of the tile sees; the others are zero.
template <int D, int NST, bool ONCE, int KINDS>
__device__ __forceinline__ unsigned move_slab(const PagedArgs& a, const Unit& u, int k, int id, int kind, unsigned lds_slab,
                                              unsigned char* slab_ptr, unsigned kg, unsigned vg) {
  using S = TileShape<D, NST>;
  // byte offset of the lane's (swizzled) 16 bytes of transfer j within the slab, less j KiB; made where they are used, of two
  // registers that the compiler cannot see through: kept over the loop they cost eight
  asm volatile("" : "+v"(kg), "+v"(vg));
  const unsigned kgj[4] = {kg, kg ^ 64, kg ^ 128, kg ^ 192};
  const unsigned vodd = D == 128 ? vg ^ 128 : vg;
  const unsigned vgj[4] = {vg, vodd, vg, vodd};
  const Seen& s = u.s;
  const int lane = threadIdx.x & 63;
  const bool valid = (unsigned)id < (unsigned)a.n_pages;
  const long long row0 = (((long long)id * a.Hkv + u.kvh) << a.shift) + (k & ((1 << a.shift) - 1));
  if (valid && k + 16 <= s.n && ((k >= s.lo && k + 16 <= s.hi) || k + 16 <= s.sink)) {
    if (KINDS == 2 || kind == 0) dma_slab<S::IPT, ONCE>(lds_slab, uniform_ptr((const unsigned char*)a.kp + row0 * S::ROWB), kgj);
    if (KINDS == 2 || kind == 1) dma_slab<S::IPT, ONCE>(lds_slab + S::VB, uniform_ptr((const unsigned char*)a.vp + row0 * S::ROWB), vgj);
    return 0xffffu;
  }
  // 16 rows of the block, all of them seen
  if (k >= s.n && k >= s.lo && k + 16 <= s.hi && a.kb_st[2] == D && a.vb_st[2] == D) {
    const long long x = k - s.n;
    if (KINDS == 2 || kind == 0)
      dma_slab<S::IPT, ONCE>(lds_slab, uniform_ptr((const unsigned char*)a.kb + 2 * (u.b * a.kb_st[0] + u.kvh * a.kb_st[1] + x * D)), kgj);
    if (KINDS == 2 || kind == 1)
      dma_slab<S::IPT, ONCE>(lds_slab + S::VB, uniform_ptr((const unsigned char*)a.vb + 2 * (u.b * a.vb_st[0] + u.kvh * a.vb_st[1] + x * D)), vgj);
    return 0xffffu;
  }
  // a border of what is seen, the end of the cache, a page that is not there: row by row, and zeros where there is no key
  const int key = k + (lane & 15);
  const bool seen = (key < s.hi) & ((key >= s.lo) | (key < s.sink)) & ((key >= s.n) | valid);
  const unsigned bits = (unsigned)__ballot(seen) & 0xffffu;
#pragma unroll
  for (int t = 0; t < S::IPT; ++t) {
    if (KINDS == 2 || kind == 0) *reinterpret_cast<u32x4*>(slab_ptr + 1024 * t + 16 * lane) = u32x4{0, 0, 0, 0};
    if (KINDS == 2 || kind == 1) *reinterpret_cast<u32x4*>(slab_ptr + S::VB + 1024 * t + 16 * lane) = u32x4{0, 0, 0, 0};
  }
  wait_lds();
#pragma unroll
  for (int t = 0; t < S::IPT; ++t) {
    const int r = S::RPI * t + lane / S::CPR;
    if ((bits >> r) & 1) {
      // kgj holds row, chunk and minus t KiB; the row is taken off again: it may lie elsewhere
      const int kc = kgj[t] + 1024 * t - r * S::ROWB, vc = vgj[t] + 1024 * t - r * S::ROWB;
      const unsigned char *kr, *vr;
      if (k + r < s.n) {
        kr = (const unsigned char*)a.kp + (row0 + r) * S::ROWB;
        vr = (const unsigned char*)a.vp + (row0 + r) * S::ROWB;
      } else {
        const long long x = k + r - s.n;
        kr = (const unsigned char*)a.kb + 2 * (u.b * a.kb_st[0] + u.kvh * a.kb_st[1] + x * a.kb_st[2]);
        vr = (const unsigned char*)a.vb + 2 * (u.b * a.vb_st[0] + u.kvh * a.vb_st[1] + x * a.vb_st[2]);
      }
      if (KINDS == 2 || kind == 0) dma16_vaddr<ONCE>(lds_slab + 1024 * t, kr + kc);
      if (KINDS == 2 || kind == 1) dma16_vaddr<ONCE>(lds_slab + S::VB + 1024 * t, vr + vc);
    }
  }
  return bits;
}

__device__ __forceinline__ int page_id(const PagedArgs& a, const Unit& u, int k) {
  const const_i32_ptr row = (const_i32_ptr)(uintptr_t)(a.table + (long long)u.b * a.max_pages);
  return row[min(k >> a.shift, a.max_pages - 1)];
}

// What a wave keeps over the tiles of a unit
template <int D, int RB> struct Rows {
  static constexpr int NS = D / 32, NDB = D / 16;
  bf16x8 q[RB][NS];                                // MFMA B operands (lane: row l16, d = 32 s + 8 G .. + 7)
  f32x4 o[RB][NDB];
  f32x4 neg_m[RB];                                 // minus the reference of row l16, four times
  float thr[RB], lsum[RB];                         // thr kNegBig: no reference yet; lsum: RB == 1 the row's, else this lane's part
  int lo[RB], hi[RB];                              // keys that row l16 sees
};

// One key tile; kro, vro: LDS offsets of the lane's first operands in the tile's ring stage
template <int D, int RB, int NST>
__device__ __forceinline__ void compute_tile(const PagedArgs& a, Rows<D, RB>& w, const unsigned char* lds, unsigned kro, unsigned vro, unsigned vtile, int k0, bool masked, bool rows_differ, u32x4 vbits) {
  using S = TileShape<D, NST>;
  constexpr int NS = S::NS, NDB = S::NDB;
  const int G = (threadIdx.x & 63) >> 4;
  auto read_vt = [&](int db, int u) {
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(lds + (vro ^ (db << 5)) + 32 * u * S::ROWB));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(lds + (vro ^ (db << 5)) + (32 * u + 16) * S::ROWB));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // ---- S^T = K Q^T - reference
  f32x4 sacc[RB][4];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) sacc[rb][kb] = w.neg_m[rb];
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int s2 = 0; s2 < NS; ++s2) {
      const bf16x8 kop = *reinterpret_cast<const bf16x8*>(lds + (kro ^ (s2 << 6)) + kb * S::SLABB);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sacc[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop, w.q[rb][s2], sacc[rb][kb], 0, 0, 0);
    }
  if (masked) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = k0 + 16 * kb + 4 * G + e;
          const bool see = ((vbits[kb] >> (4 * G + e)) & 1) & (key < w.hi[rb]) & ((key >= w.lo[rb]) | (key < a.sinks));
          sacc[rb][kb][e] = see ? sacc[rb][kb][e] : -INFINITY;
        }
  }
  // ---- online softmax
  s16x8 pk[RB][2];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float mx = fmaxf(fmaxf(sacc[rb][0][0], sacc[rb][0][1]), sacc[rb][0][2]);
    mx = fmaxf(fmaxf(mx, sacc[rb][0][3]), sacc[rb][1][0]);
    mx = fmaxf(fmaxf(mx, sacc[rb][1][1]), sacc[rb][1][2]);
    mx = fmaxf(fmaxf(mx, sacc[rb][1][3]), sacc[rb][2][0]);
    mx = fmaxf(fmaxf(mx, sacc[rb][2][1]), sacc[rb][2][2]);
    mx = fmaxf(fmaxf(mx, sacc[rb][2][3]), sacc[rb][3][0]);
    mx = fmaxf(fmaxf(mx, sacc[rb][3][1]), sacc[rb][3][2]);
    mx = fmaxf(mx, sacc[rb][3][3]);
    if (__builtin_amdgcn_ballot_w64(mx > w.thr[rb]) != 0) {
      const auto s16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(s16[0]), __uint_as_float(s16[1]));
      const auto s32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(s32[0]), __uint_as_float(s32[1]));
      const bool move = mx > w.thr[rb];
      const float shift = move ? mx : 0.f;
      const float corr = w.thr[rb] == kNegBig ? 0.f : exp2_fast(-shift * a.scale_log2);
      w.lsum[rb] *= corr;
#pragma unroll
      for (int db = 0; db < NDB; ++db) w.o[rb][db] *= corr;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) sacc[rb][kb] -= shift;
      w.neg_m[rb] -= shift;
      w.thr[rb] = move ? a.thr8 : w.thr[rb];
    }
    float ps = 0.f;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = exp2_fast(sacc[rb][kb][e] * a.scale_log2);
        sacc[rb][kb][e] = p;
        if (RB != 1) ps += p;
      }
    if (RB != 1) w.lsum[rb] += ps;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      union { uint32_t x[4]; s16x8 v; } cv;
      cv.x[0] = pack_bf16x2(sacc[rb][2 * u][0], sacc[rb][2 * u][1]);
      cv.x[1] = pack_bf16x2(sacc[rb][2 * u][2], sacc[rb][2 * u][3]);
      cv.x[2] = pack_bf16x2(sacc[rb][2 * u + 1][0], sacc[rb][2 * u + 1][1]);
      cv.x[3] = pack_bf16x2(sacc[rb][2 * u + 1][2], sacc[rb][2 * u + 1][3]);
      pk[rb][u] = cv.v;
    }
  }
  if (RB == 1) {                                   // row sums on the matrix pipe, as in the dense kernel
    union { uint32_t x[4]; s16x8 v; } ones;
    ones.x[0] = ones.x[1] = ones.x[2] = ones.x[3] = 0x3f803f80u;
    f32x4 ls = {w.lsum[0], 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 2; ++u)
      ls = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones.v), __builtin_bit_cast(bf16x8, pk[0][u]), ls, 0, 0, 0);
    w.lsum[0] = ls[0];
  }
  // ---- O^T += V^T P^T
  if (masked && rows_differ) {                     // what a row does not see must not reach it
    const int lane = threadIdx.x & 63;
    bool bad = false;
#pragma unroll 4
    for (int it = 0; it < S::STAGEB / 1024; ++it) bad |= has_nonfinite(*reinterpret_cast<const u32x4*>(lds + vtile + 1024 * it + 16 * lane));
    if (__builtin_expect(__ballot(bad) != 0, 0)) {
#pragma unroll 1
      for (int kind = 0; kind < 3; ++kind)
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          asm volatile("" ::: "memory");           // keeps the reads where they are: all of them at once do not fit the registers
          const s16x8 v0 = is_kind(read_vt(db, 0), kind), v1 = is_kind(read_vt(db, 1), kind);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v0), __builtin_bit_cast(bf16x8, weighed(pk[rb][0])), c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v1), __builtin_bit_cast(bf16x8, weighed(pk[rb][1])), c, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) w.o[rb][db][e] += c[e] != 0.f ? of_kind(kind) : 0.f;
          }
        }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          asm volatile("" ::: "memory");
          const s16x8 vop = finite_part(read_vt(db, u));
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            w.o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vop), __builtin_bit_cast(bf16x8, pk[rb][u]), w.o[rb][db], 0, 0, 0);
        }
      return;
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      const s16x8 vop = read_vt(db, u);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        w.o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vop), __builtin_bit_cast(bf16x8, pk[rb][u]), w.o[rb][db], 0, 0, 0);
    }
}

template <int D, int RB, int NW, bool FLAT>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void paged_tile_kernel(PagedArgs a) {
  constexpr int NST = 2, WROWS = 16 * RB, KINDS = NW == 8 ? 1 : 2;
  constexpr bool ONCE = FLAT;                      // K/V is read by one workgroup only
  using S = TileShape<D, NST>;
  constexpr int CPR = S::CPR, R256 = S::R256, NS = S::NS, NDB = S::NDB, ROWB = S::ROWB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  u32x4* vis_s = reinterpret_cast<u32x4*>(lds + 2 * NST * S::STAGEB);      // per stage: rows of the four slabs that hold a key
  const int lane = threadIdx.x & 63, l16 = lane & 15, G = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6), slab = wave & 3, kind = wave >> 2;

  // ---- this workgroup's tiles
  Unit nxt;
  long long f, f1, slot_unit = 0;
  int row_base = 0;
  if constexpr (FLAT) {
    if (a.min_tiles == 0) {                        // a workgroup per (sequence, K/V head)
      open_unit<kTK>(a, nxt, blockIdx.x / a.Hkv, blockIdx.x % a.Hkv, 0);
      f = 0; f1 = nxt.T;
    } else {
      const long long total = all_tiles<kTK>(a), per = tiles_per_worker(a, total);
      f = blockIdx.x * per; f1 = f + per < total ? f + per : total;
      if (f >= f1) return;
      locate<kTK>(a, f, nxt);
    }
  } else {
    const unsigned units = (unsigned)(a.B * a.Hkv * a.parts);
    const int rank = blockIdx.x / units, unit = blockIdx.x - rank * units;
    const int part = unit % a.parts, bh = unit / a.parts;
    nxt.b = bh / a.Hkv; nxt.kvh = bh - nxt.b * a.Hkv;
    row_base = (a.row_tiles - 1 - rank) * (WROWS * NW);
    const int r0 = row_base / a.g, r1 = (row_base + WROWS * NW - 1) / a.g;
    nxt.s = seen_by(a, a.lens[nxt.b], a.q_lens ? a.q_lens[nxt.b] : a.K, r0, r1, kTK);
    nxt.T = row_base < nxt.s.q_len * a.g ? max(nxt.s.tiles, 1) : 0;
    const int per = max((nxt.T + a.parts - 1) / a.parts, a.min_tiles);
    nxt.i = part * per;
    f = nxt.i; f1 = min(nxt.i + per, nxt.T);
    slot_unit = (long long)bh * a.parts + part;
  }
  if (f >= f1) return;

  // LDS and source offsets of a lane; the others differ in bits that a slice, a block, a transfer number flips
  const int row = lane / CPR, chunk = lane % CPR;
  const unsigned kg = row * ROWB + ((chunk ^ ((row / R256) % CPR)) << 4), vg = row * ROWB + ((chunk ^ (2 * ((row / R256) % (CPR / 2)))) << 4);
  unsigned kro, vro;                               // operands of slice 0 / d block 0 in the current ring stage
  {
    kro = l16 * ROWB + ((G ^ ((D == 128) ? l16 : (l16 >> 1))) << 4);
    const int e4 = l16 >> 2, c4 = l16 & 3;
    const int fv = (D == 128) ? 2 * (4 * (G & 1) + e4) : 2 * (2 * (G & 1) + (e4 >> 1));
    vro = S::VB + (4 * G + e4) * ROWB + (((c4 >> 1) ^ fv) << 4) + ((c4 & 1) << 3);
  }
  const unsigned lds_slab = uniform((int)(unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)lds) + slab * S::SLABB;

  // tile of the unit at nxt into ring stage `stage`; `id`: the page of the wave's slab, the next tile's on return
  auto issue = [&](int stage, int& id) {
    unsigned bits = 0;
    if (nxt.s.tiles > 0)
      bits = move_slab<D, NST, ONCE, KINDS>(a, nxt, nxt.s.tile(nxt.i) * kTK + 16 * slab, id, kind, lds_slab + stage * S::STAGEB,
                                            lds + slab * S::SLABB + stage * S::STAGEB, kg, vg);
    if (kind == 0 && lane == 0) reinterpret_cast<unsigned*>(vis_s + stage)[slab] = bits;
    id = page_id(a, nxt, nxt.s.tile(min(nxt.i + 1, nxt.T - 1)) * kTK + 16 * slab);
  };
  int id = page_id(a, nxt, nxt.s.tile(nxt.i) * kTK + 16 * slab);
  issue(0, id);

  int stage = 0, part_slot = 0;
  while (f < f1) {
    // ---- a unit
    const Unit cur = nxt;
    const int begin = cur.i, last_row = cur.s.q_len * a.g - 1;
    const int wave_row = row_base + wave * WROWS;
    const bool has_rows = wave_row <= last_row;
    Rows<D, RB> w;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int R = min(wave_row + 16 * rb + l16, last_row), r = R / a.g, h = cur.kvh * a.g + R - r * a.g;
      const uint16_t* qp = (const uint16_t*)a.q + cur.b * a.q_st[0] + h * a.q_st[1] + r * a.q_st[2];
#pragma unroll
      for (int s2 = 0; s2 < NS; ++s2) w.q[rb][s2] = *reinterpret_cast<const bf16x8*>(qp + 32 * s2 + 8 * G);
      row_range(a, cur.s, r, w.lo[rb], w.hi[rb]);
      w.neg_m[rb] = f32x4{0.f, 0.f, 0.f, 0.f}; w.thr[rb] = kNegBig; w.lsum[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < NDB; ++db) w.o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // what the wave's rows see: all of them [all_lo, all_hi), any of them [any_lo, any_hi)
    const int r0 = min(wave_row, last_row) / a.g, r1 = min(wave_row + WROWS - 1, last_row) / a.g;
    int any_lo, all_hi, all_lo, any_hi;
    row_range(a, cur.s, r0, any_lo, all_hi);
    row_range(a, cur.s, r1, all_lo, any_hi);
    int i = begin;
    while (i < cur.T && f < f1) {
      wait_transfers();
      wait_lds();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const bool more = f + 1 < f1;
      const u32x4 seen = vis_s[stage];
      if (more) {
        if constexpr (FLAT) {
          next_tile<kTK>(a, nxt);
          if (nxt.i == 0) id = page_id(a, nxt, nxt.s.tile(0) * kTK + 16 * slab);
        } else {
          ++nxt.i;
        }
        issue(stage ^ 1, id);
      }
      const int k0 = cur.s.tile(i) * kTK;
      const u32x4 vb{(unsigned)uniform(seen[0]), (unsigned)uniform(seen[1]), (unsigned)uniform(seen[2]), (unsigned)uniform(seen[3])};
      const bool any = (vb[0] | vb[1] | vb[2] | vb[3]) != 0, all = (vb[0] & vb[1] & vb[2] & vb[3]) == 0xffffu;
      if (has_rows && any && k0 < any_hi && (k0 + kTK > any_lo || k0 < a.sinks)) {
        const bool masked = !all || k0 + kTK > all_hi || (k0 < all_lo && k0 + kTK > a.sinks);
        compute_tile<D, RB, NST>(a, w, lds, kro, vro, S::VB + stage * S::STAGEB, k0, masked, r1 > r0, vb);
      }
      ++i; ++f;
      stage ^= 1;
      kro ^= S::STAGEB;                            // (bits below a stage's size are those within a tile)
      vro ^= S::STAGEB;
    }

    // ---- this workgroup's share of the unit is done
    const bool whole = begin == 0 && i == cur.T;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float l = w.lsum[rb];
      if (RB != 1) {
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
      }
      const int R = wave_row + 16 * rb + l16;
      if (R > last_row) continue;
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const int r = R / a.g, h = cur.kvh * a.g + R - r * a.g;
        uint16_t* orow = (uint16_t*)a.out + cur.b * a.o_st[0] + h * a.o_st[1] + r * a.o_st[2];
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          uint2 x;
          x.x = pack_bf16x2(w.o[rb][db][0] * inv, w.o[rb][db][1] * inv);
          x.y = pack_bf16x2(w.o[rb][db][2] * inv, w.o[rb][db][3] * inv);
          *reinterpret_cast<uint2*>(orow + 16 * db + 4 * G) = x;
        }
      } else {
        const long long slot = (FLAT ? (long long)blockIdx.x * 2 + part_slot : slot_unit) * a.R + R;
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4*>(a.ws_o + slot * D + 16 * db + 4 * G) = w.o[rb][db];
        if (G == 0) { a.ws_ml[2 * slot] = w.thr[rb] == kNegBig ? kNegBig : -w.neg_m[rb][0]; a.ws_ml[2 * slot + 1] = l; }
      }
    }
    part_slot = 1;
  }
}

// Merges the parts of a row that a row tile's workgroups left, in the order of the keys: D / 4 lanes per row
template <int D>
__global__ __launch_bounds__(256) void paged_parts_merge_kernel(PagedArgs a, int rows_wg) {
  constexpr int TPR = D / 4, RPB = 256 / TPR;
  const long long at = (long long)blockIdx.x * RPB + threadIdx.x / TPR;
  if (at >= (long long)a.B * a.Hkv * a.R) return;
  const int bh = (int)(at / a.R), R = (int)(at - (long long)bh * a.R), b = bh / a.Hkv, kvh = bh - b * a.Hkv;
  const int base = R / rows_wg * rows_wg;
  const Seen s = seen_by(a, a.lens[b], a.q_lens ? a.q_lens[b] : a.K, base / a.g, (base + rows_wg - 1) / a.g, kTK);
  if (R >= s.q_len * a.g) return;
  const int T = max(s.tiles, 1), per = max((T + a.parts - 1) / a.parts, a.min_tiles), n = (T + per - 1) / per;
  if (n == 1) return;                              // written by its workgroup
  const int d = (threadIdx.x % TPR) * 4;
  float M = kNegBig, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < n; ++k) {
    const long long slot = ((long long)bh * a.parts + k) * a.R + R;
    const f32x4 ov = *reinterpret_cast<const f32x4*>(a.ws_o + slot * D + d);
    const float mk = a.ws_ml[2 * slot], lk = a.ws_ml[2 * slot + 1];
    const float up = fmaxf(M, mk), c0 = exp2_fast((M - up) * a.scale_log2), c1 = exp2_fast((mk - up) * a.scale_log2);
    acc = acc * c0 + ov * c1;
    l = l * c0 + lk * c1;
    M = up;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int r = R / a.g, h = kvh * a.g + R - r * a.g;
  uint2 w2;
  w2.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  w2.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<uint2*>((uint16_t*)a.out + b * a.o_st[0] + h * a.o_st[1] + r * a.o_st[2] + d) = w2;
}

// ---- launch plan, from the parameters alone
struct TilePlan { int rb, waves, flat, workers, parts, row_tiles, min_tiles; };

static TilePlan plan_tile(const sdllm_paged_attn_params& p, bool with_block) {
  const long long R = (long long)p.Hq / p.Hkv * p.K, units = (long long)p.B * p.Hkv;
  const long long N = p.max_kv_len + (with_block ? p.K : 0);
  TilePlan pl{};
  pl.waves = R > 128 ? 8 : 4;
  pl.rb = R > 64 ? 2 : 1;
  const int rows = 16 * pl.rb * pl.waves;
  pl.row_tiles = (int)((R + rows - 1) / rows);
  pl.flat = pl.row_tiles == 1 && p.B <= 1024;
  long long tiles = (N + kTK - 1) / kTK;
  if (p.window > 0) {
    const long long span = (rows + p.Hq / p.Hkv - 1) / (p.Hq / p.Hkv);
    const long long seen = (p.window + (span < p.K ? span : p.K) + kTK - 2) / kTK + 1 + (p.sinks + kTK - 1) / kTK;
    if (seen < tiles) tiles = seen;
  }
  if (tiles < 1) tiles = 1;
  const long long at_once = (pl.waves == 8 ? 1 : 2) * kNumCUs;
  pl.min_tiles = 2;
  if (p.kv_splits > 0) pl.min_tiles = (int)((tiles + p.kv_splits - 1) / p.kv_splits);
  if (pl.flat) {
    pl.parts = 1;
    if (p.kv_splits == 1 || (p.kv_splits == 0 && (units >= 4 * at_once || tiles <= pl.min_tiles))) {
      pl.workers = (int)units; pl.min_tiles = 0;
      return pl;
    }
    const long long w = (units * tiles + pl.min_tiles - 1) / pl.min_tiles;
    pl.workers = (int)(p.kv_splits > 0 ? (w < (1 << 20) ? w : 1 << 20) : (w < at_once ? w : at_once));
    return pl;
  }
  long long parts = p.kv_splits > 0 ? p.kv_splits : at_once / (units * pl.row_tiles);
  const long long most = (tiles + pl.min_tiles - 1) / pl.min_tiles;
  if (parts > most) parts = most;
  if (parts < 1) parts = 1;
  pl.parts = (int)parts;
  return pl;
}

size_t paged_tile_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  const TilePlan pl = plan_tile(p, with_block);
  const size_t R = (size_t)(p.Hq / p.Hkv) * p.K;
  if (pl.flat) return pl.min_tiles == 0 ? 0 : (size_t)pl.workers * 2 * R * (p.D + 2) * sizeof(float);
  return pl.parts == 1 ? 0 : (size_t)p.B * p.Hkv * pl.parts * R * (p.D + 2) * sizeof(float);
}

template <int D, int RB, int NW, bool FLAT>
static hipError_t launch_tile(const PagedArgs& a, unsigned grid, hipStream_t stream, bool launch) {
  constexpr size_t bytes = TileShape<D, 2>::LDS;
  static LdsOptIn st;
  hipError_t e = ensure_lds_opt_in(reinterpret_cast<const void*>(&paged_tile_kernel<D, RB, NW, FLAT>), bytes, st);
  if (e != hipSuccess || !launch) return e;
  hipLaunchKernelGGL((paged_tile_kernel<D, RB, NW, FLAT>), dim3(grid), dim3(64 * NW), bytes, stream, a);
  return hipGetLastError();
}
template <int D>
static hipError_t launch_tile_d(const PagedArgs& a, const TilePlan& pl, unsigned grid, hipStream_t stream, bool launch = true) {
  if (pl.waves == 8) return pl.flat ? launch_tile<D, 2, 8, true>(a, grid, stream, launch) : launch_tile<D, 2, 8, false>(a, grid, stream, launch);
  if (pl.rb == 2) return pl.flat ? launch_tile<D, 2, 4, true>(a, grid, stream, launch) : launch_tile<D, 2, 4, false>(a, grid, stream, launch);
  return pl.flat ? launch_tile<D, 1, 4, true>(a, grid, stream, launch) : launch_tile<D, 1, 4, false>(a, grid, stream, launch);
}

hipError_t prepare_paged_tile() {
  hipError_t e = hipSuccess;
  for (int waves = 4; waves <= 8; waves += 4)
    for (int rb = 1; rb <= 2; ++rb)
      for (int flat = 0; flat <= 1; ++flat) {
        TilePlan pl{};
        pl.waves = waves; pl.rb = rb; pl.flat = flat;
        if (e == hipSuccess) e = launch_tile_d<64>(PagedArgs{}, pl, 0, nullptr, false);
        if (e == hipSuccess) e = launch_tile_d<128>(PagedArgs{}, pl, 0, nullptr, false);
      }
  return e;
}

hipError_t launch_paged_tile(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream) {
  const TilePlan pl = plan_tile(p, a.kb != nullptr);
  a.workers = pl.workers; a.min_tiles = pl.min_tiles; a.parts = pl.parts; a.row_tiles = pl.row_tiles;
  const bool merge = pl.flat ? pl.min_tiles > 0 : pl.parts > 1;
  const size_t slots = pl.flat ? (size_t)pl.workers * 2 : (size_t)p.B * p.Hkv * pl.parts;
  a.ws_o = merge ? (float*)workspace : nullptr;
  a.ws_ml = merge ? a.ws_o + slots * a.R * p.D : nullptr;
  const unsigned grid = pl.flat ? (unsigned)pl.workers : (unsigned)((long long)p.B * p.Hkv * pl.parts * pl.row_tiles);
  hipError_t e = p.D == 128 ? launch_tile_d<128>(a, pl, grid, stream) : launch_tile_d<64>(a, pl, grid, stream);
  if (e != hipSuccess || !merge) return e;
  if (pl.flat) return launch_shares_merge(a, p.D, kTK, stream);
  const int rows_wg = 16 * pl.rb * pl.waves, rpb = 256 / (p.D / 4);
  const unsigned blocks = (unsigned)(((long long)a.B * a.Hkv * a.R + rpb - 1) / rpb);
  if (p.D == 128) hipLaunchKernelGGL(paged_parts_merge_kernel<128>, dim3(blocks), dim3(256), 0, stream, a, rows_wg);
  else hipLaunchKernelGGL(paged_parts_merge_kernel<64>, dim3(blocks), dim3(256), 0, stream, a, rows_wg);
  return hipGetLastError();
}

}  // namespace sdllm
