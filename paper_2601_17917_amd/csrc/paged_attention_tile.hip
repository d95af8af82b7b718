// bf16 attention over a paged K/V cache for gfx950 (sdllm_paged_attention), more than 32 query rows per (sequence, K/V head): the
// rows of a block over its heads, the pieces of prompts.
//
// A workgroup owns 16 RB NW query rows (NW waves, 16 RB rows each) and walks key tiles of 64 that its waves share through a
// ring in LDS: each wave moves 16-row slabs global -> LDS, one tile ahead of the one being computed (four waves, two workgroups per CU)
// or two (eight waves, one workgroup per CU), one barrier per tile.  Products, operand layouts and the softmax are those of the stream kernel, but
// for the weights of the values: rounded to bf16 (2^-8), as in the dense kernel, and divided by the sum of the rounded ones.  Here the matrix
// unit is the bound; a second number for what the rounding takes cost 8 sequences of 500 to 8000 keys (28 / 4 heads, 32 rows) 34 -> 39 us and
// 2 x 2048 causal rows behind up to 4096 keys 203 -> 281.
//   FLAT (four waves of 16 rows): one row tile covers a (sequence, K/V head).  The workgroups walk equal shares of all key tiles of
//         the call, laid end to end as the stream kernel's waves do, so that lengths need not be alike.
//   else: a workgroup per (row tile, sequence, K/V head), the tiles of the last rows, which see most under a causal mask, first; or,
//         where that is fewer than fit on the chip, per (row tile, sequence, K/V head, part of the keys).  Sequences get parts by their
//         lengths: parts have as few tiles as let all workgroups be on the chip at once.
// Many rows are bound by the matrix cores and the softmax between them: 8 x 512 rows of 32 / 8 heads over 4096 keys 250 us (1.10
// PFLOP/s), 2 x 2048 causal rows behind 4096 keys 303 us (1.13).  Blocks, 28 and 4 heads of 32 rows, 8 sequences of 500 to 8000 keys: 27 us
// and 8 us in the merge, of which a workgroup's start (its place, table, queries, the first two tiles) and end are 10.
#include "paged_attention.h"
#include <algorithm>

namespace sdllm {

constexpr int kTK = 64;                            // keys per tile
typedef const bf16x8 __attribute__((address_space(3))) * lds_bf16x8_ptr;
typedef u32x4 __attribute__((address_space(3))) * lds_u32x4_ptr;
typedef int __attribute__((address_space(3))) * lds_int_ptr;

template <int D, int NST> struct TileShape {
  static constexpr int NS = D / 32, NDB = D / 16, ROWB = D * 2;
  static constexpr int SLABB = 16 * ROWB, STAGEB = kTK * ROWB, VB = NST * STAGEB, FLAG = 2 * NST * STAGEB, LDS = FLAG + 16;
};

// What a wave keeps over the tiles of a unit
template <int D, int RB> struct Rows {
  static constexpr int NS = D / 32, NDB = D / 16;
  bf16x8 q[RB][NS];                                // MFMA B operands (lane: row l16, d = 32 s + 8 G .. + 7)
  f32x4 o[RB][NDB];
  float neg_m[RB];                                 // minus the reference of row l16
  float thr[RB], lsum[RB];                         // thr kNegBig: no reference yet
  int pos[RB];                                     // position of row l16
};

// One key tile.  kro, vro: LDS addresses of the lane's first operands in the tile's ring stage
template <int D, int RB, int NST>
__device__ __forceinline__ void compute_tile(const Hot& h, Rows<D, RB>& w, unsigned kro, unsigned vro, int k0, bool missing, bool above,
                                             bool below, unsigned long long vis) {
  using S = TileShape<D, NST>;
  constexpr int NS = S::NS, NDB = S::NDB;
  auto read_vt = [&](int db, int u) {
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)((vro ^ (db << 5)) + 32 * u * S::ROWB));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)((vro ^ (db << 5)) + (32 * u + 16) * S::ROWB));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // ---- S^T = K Q^T - reference
  f32x4 sacc[RB][4];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) sacc[rb][kb] = f32x4{w.neg_m[rb], w.neg_m[rb], w.neg_m[rb], w.neg_m[rb]};
  // all operand reads first, so that the products find theirs in registers one after the other (memory operations and products stay on
  // their side of these barriers, other arithmetic need not)
  bf16x8 kop[4][NS];
#pragma unroll
  for (int s2 = 0; s2 < NS; ++s2)
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) kop[kb][s2] = *(lds_bf16x8_ptr)(uintptr_t)((kro ^ (s2 << 6)) + kb * S::SLABB);
  __builtin_amdgcn_sched_barrier(0x406);
#pragma unroll
  for (int s2 = 0; s2 < NS; ++s2)
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sacc[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[kb][s2], w.q[rb][s2], sacc[rb][kb], 0, 0, 0);
  // the values of the tile's first half travel under the softmax
  s16x8 vop[2][NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) vop[0][db] = read_vt(db, 0);
  __builtin_amdgcn_sched_barrier(0x406);
  if (missing || above || below) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) hide<4>(sacc[rb], k0, w.pos[rb] - h.window + 1, w.pos[rb] + 1, h.sinks, vis, missing, above, below);
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
      const float corr = w.thr[rb] == kNegBig ? 0.f : exp2_fast(-shift * h.scale_log2);
      w.lsum[rb] *= corr;
#pragma unroll
      for (int db = 0; db < NDB; ++db) w.o[rb][db] *= corr;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) sacc[rb][kb] -= shift;
      w.neg_m[rb] -= shift;
      w.thr[rb] = move ? h.thr8 : w.thr[rb];
    }
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) sacc[rb][kb][e] = exp2_fast(sacc[rb][kb][e] * h.scale_log2);
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
  // row sums on the matrix pipe, from the rounded weights that the values are multiplied by
  union { uint32_t x[4]; s16x8 v; } ones;
  ones.x[0] = ones.x[1] = ones.x[2] = ones.x[3] = 0x3f803f80u;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    f32x4 ls = {w.lsum[rb], 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 2; ++u)
      ls = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones.v), __builtin_bit_cast(bf16x8, pk[rb][u]), ls, 0, 0, 0);
    w.lsum[rb] = ls[0];
  }
  // ---- O^T += V^T P^T
#pragma unroll
  for (int db = 0; db < NDB; ++db) vop[1][db] = read_vt(db, 1);
  __builtin_amdgcn_sched_barrier(0x406);
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
        w.o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vop[u][db]), __builtin_bit_cast(bf16x8, pk[rb][u]), w.o[rb][db], 0, 0, 0);
}

// ---- Parts: u counts (sequence, part, K/V head) over the call.
// Tiles that decide on the number of parts of sequence b: of its first or its last row tile, whichever has more
__device__ __forceinline__ int tiles_of_sequence(Args a, int b, int& n, int& q_len) {
  n = q_len = 0;
  if (b >= a->B) return 0;
  n = a->lens[b];
  q_len = min(max(a->q_lens ? a->q_lens[b] : a->K, 0), a->K);
  if (q_len == 0) return 0;
  const int last = divide(q_len * a->g - 1, a->by_tile_rows);
  return max(tiles_to_do(a, entry_seen<kTK>(a, n, q_len, 0), 0), tiles_to_do(a, entry_seen<kTK>(a, n, q_len, last), last));
}
struct Part { int b, kvh, index, n, len, q_len; }; // part `index` of n of a sequence
// Number u0 of the first of a sequence's parts, for u >= 0 of the sequence that u belongs to, else of sequence p.b; false: none
__device__ __forceinline__ bool find_part(int u, Part& p, int& u0) {
  const Args a = arguments();
  const int lane = threadIdx.x & 63;
  int len, q_len, unused[2];
  int t = tiles_of_sequence(a, lane, len, q_len);
  long long total = read_lane(wave_scan(t), 63);
  for (int b0 = 64; b0 < a->B; b0 += 64) total += read_lane(wave_scan(tiles_of_sequence(a, b0 + lane, unused[0], unused[1])), 63);
  // Tiles of a part: so many that there are no more parts than workers (one to a K/V head and sequence always fits)
  int per = (int)tiles_per_worker(a, total * a->Hkv);
  while (true) {
    long long n = read_lane(wave_scan((t + per - 1) / per), 63);
    for (int b0 = 64; b0 < a->B; b0 += 64) n += read_lane(wave_scan((tiles_of_sequence(a, b0 + lane, unused[0], unused[1]) + per - 1) / per), 63);
    if (n * a->Hkv <= a->workers) break;
    per += per / 8 + 1;
  }
  u0 = 0;
  for (int b0 = 0; b0 < a->B; b0 += 64) {
    if (b0 > 0) t = tiles_of_sequence(a, b0 + lane, len, q_len);
    const int n = (t + per - 1) / per, upto = wave_scan(n * a->Hkv), all = read_lane(upto, 63);
    if (u >= 0 ? u < u0 + all : p.b < b0 + 64) {
      const int l = u >= 0 ? __builtin_ctzll(__ballot(upto > u - u0)) : p.b - b0;
      p.b = b0 + l;
      p.n = read_lane(n, l); p.len = read_lane(len, l); p.q_len = read_lane(q_len, l);
      u0 += read_lane(upto, l) - p.n * a->Hkv;
      if (u >= 0) { p.index = divide(u - u0, a->by_Hkv); p.kvh = u - u0 - p.index * a->Hkv; }
      return true;
    }
    u0 += all;
  }
  return false;
}

template <int D, int RB, int NW, bool FLAT>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_tile_kernel(PagedArgs) {
  constexpr int NST = NW == 8 ? 3 : 2, WROWS = 16 * RB;
  constexpr bool ONCE = FLAT;                      // K/V is read by one workgroup only
  using S = TileShape<D, NST>;
  constexpr int NS = S::NS, NDB = S::NDB, ROWB = S::ROWB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int lane = threadIdx.x & 63, l16 = lane & 15, G = lane >> 4;
  const int wave = uniform(threadIdx.x >> 6);
  const int slab = wave & 3, kind = wave >> 2;     // four waves move K and V of a slab each, eight one of the two

  // ---- this workgroup's tiles
  const Hot h = hot_arguments();
  Pages pages;
  Unit nxt;
  int left, row_base = 0;                          // tiles still to do; first query row
  long long slot = 2LL * blockIdx.x;               // of its partial results
  {
    const Args a = arguments();
    if constexpr (FLAT) {
      if (a->min_tiles == 0) {                     // a workgroup per (sequence, K/V head)
        open_whole_unit<kTK>(nxt, pages, h, blockIdx.x);
        left = nxt.T;
      } else {
        left = open_share<kTK>(blockIdx.x, nxt);
        pages.open(nxt.b);
      }
    } else {
      // The row tiles of a (sequence, K/V head, part) run one after the other on one XCD, whose L2 brings them K and V once
      const int xcd = blockIdx.x % kNumXCDs, at = blockIdx.x / kNumXCDs;
      if (a->min_tiles == 0) {
        // last rows first; heads that do not go round the XCDs evenly are cut into `cuts` lists of every so many-th row tile
        const int list = (a->row_tiles + a->cuts - 1) / a->cuts;
        const int v = at / list * kNumXCDs + xcd, bh = v / a->cuts, rank = (at % list) * a->cuts + v % a->cuts;
        if (bh >= a->B * a->Hkv || rank >= a->row_tiles) return;
        const int b = divide(bh, a->by_Hkv);
        open_whole_unit<kTK>(nxt, pages, h, (b * a->row_tiles + a->row_tiles - 1 - rank) * a->Hkv + bh - b * a->Hkv);
        left = nxt.T;
      } else {
        const int g8 = divide(at, a->by_row_tiles), rt = at - g8 * a->row_tiles, u = g8 * kNumXCDs + xcd;
        Part p;
        int u0;
        if (!find_part(u, p, u0)) return;
        pages.open(p.b);
        open_unit<kTK>(nxt, p.b * a->row_tiles + rt, p.kvh, 0, p.len, p.q_len);
        const int per = (nxt.T + p.n - 1) / p.n;
        nxt.i = p.index * per;
        left = min(per, nxt.T - nxt.i);
        slot = u;
      }
      row_base = nxt.rt * a->tile_rows;
    }
  }
  if (left <= 0) return;
  BlockRows<D> block;
  block.open(nxt.b, nxt.kvh);

  // LDS addresses of the lane's operands of slice 0 / d block 0 in stage 0; the others flip bits of them
  const unsigned lds0 = uniform((int)(unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)lds);
  const int e4 = l16 >> 2, c4 = l16 & 3, fv = (D == 128) ? 2 * (4 * (G & 1) + e4) : 2 * (2 * (G & 1) + (e4 >> 1));
  const unsigned kro = lds0 + l16 * ROWB + ((G ^ ((D == 128) ? l16 : (l16 >> 1))) << 4);
  const unsigned vro = lds0 + S::VB + (4 * G + e4) * ROWB + (((c4 >> 1) ^ fv) << 4) + ((c4 & 1) << 3);
  const unsigned lds_slab = lds0 + slab * S::SLABB;

  // Tiles of nxt's unit that start at keys [plain, plain + plain_span] are whole, cached, and in valid pages of the 64 entries at hand:
  // one comparison and an address for most tiles.  (Eight waves that each go through all the conditions below cost a tile 400 cycles.)
  int plain = 0x7fffffff;
  unsigned plain_span = 0;
  unsigned k_off[4], v_off[4];                     // the lane's offsets within a slab
  Slab<D>::offsets(false, k_off);
  Slab<D>::offsets(true, v_off);
  // Puts the tile at nxt in flight into ring stage `stage`; returns which of its keys some query row sees.  A tile that is not whole
  // has landed on return (its transfers are not counted).
  auto issue = [&](int stage) -> unsigned long long {
    const Seen& s = nxt.s;
    const int k0 = s.tile(nxt.i) * kTK, k = k0 + 16 * slab;
    const unsigned to = lds_slab + stage * S::STAGEB;
    if ((unsigned)(k0 - plain) <= plain_span) {
      const unsigned long long at = row_offset(h, pages.of(h, k), nxt.kvh, k, ROWB);
      if (NW == 4 || kind == 0) dma_slab<Slab<D>::IPT, ONCE>(to, uniform_ptr(h.kp + at), k_off);
      if (NW == 4 || kind == 1) dma_slab<Slab<D>::IPT, ONCE>(to + S::VB, uniform_ptr(h.vp + at), v_off);
      return ~0ull;
    }
    if (k0 >= s.n && k0 >= s.lo && k0 + kTK <= s.hi && block.k_stride != 0) {
      const unsigned long long x = (unsigned)(k - s.n);
      const unsigned char *kr = block.k + x * block.k_stride, *vr = block.v + x * block.v_stride;
      if (block.k_stride == ROWB && block.v_stride == ROWB) {
        if (NW == 4 || kind == 0) dma_slab<Slab<D>::IPT, ONCE>(to, uniform_ptr(kr), k_off);
        if (NW == 4 || kind == 1) dma_slab<Slab<D>::IPT, ONCE>(to + S::VB, uniform_ptr(vr), v_off);
      } else {
        if (NW == 4 || kind == 0) move_strided<D, ONCE, false>(to, kr, block.k_stride);
        if (NW == 4 || kind == 1) move_strided<D, ONCE, true>(to + S::VB, vr, block.v_stride);
      }
      return ~0ull;
    }
    pages.seek(h, k0);
    {
      const int lo = max(s.lo, pages.begin(h)), hi = min(s.last16 + 16, pages.valid_until(h)) - kTK;
      plain = hi >= lo && s.tiles > 0 ? lo : 0x7fffffff;
      plain_span = hi >= lo ? hi - lo : 0;
    }
    const unsigned long long at = row_offset(h, pages.of(h, k), nxt.kvh, k, ROWB);
    if (s.tiles > 0 && pages.all_ok<kTK>(h, k0) && ((k0 >= s.lo && k0 + kTK - 16 <= s.last16) || k0 + kTK - 16 <= s.sink16)) {
      if constexpr (NW == 8) {
        if (kind == 0) move_slab<D, ONCE, false>(to, h.kp + at);
        else move_slab<D, ONCE, true>(to + S::VB, h.vp + at);
      } else {
        move_slab<D, ONCE, false>(to, h.kp + at);
        move_slab<D, ONCE, true>(to + S::VB, h.vp + at);
      }
      return ~0ull;
    }
    const unsigned long long vis = seen_keys<kTK>(h, s, pages, k0);    // rows that see nothing: none
    const unsigned bits = (unsigned)(vis >> (16 * slab)) & 0xffffu;
    unsigned char* const ptr = lds + slab * S::SLABB + stage * S::STAGEB;
    if (NW == 4 || kind == 0) move_rows<D, ONCE, false>(s, nxt.b, nxt.kvh, k, bits, h.kp + at, to, ptr);
    if (NW == 4 || kind == 1) move_rows<D, ONCE, true>(s, nxt.b, nxt.kvh, k, bits, h.vp + at, to + S::VB, ptr + S::VB);
    if (NST > 2) wait_transfers();
    return vis;
  };
  auto advance = [&]() {                           // nxt to the next tile of the share
    if constexpr (FLAT) {
      const int b = nxt.b, kvh = nxt.kvh;
      next_tile<kTK>(nxt);
      if (nxt.b != b) pages.open(nxt.b);
      if (nxt.b != b || nxt.kvh != kvh) {
        block.open(nxt.b, nxt.kvh);
        plain = 0x7fffffff; plain_span = 0;
      }
    } else {
      ++nxt.i;
    }
  };
  // Number of the last tile of which a value was taken out (values that are not finite, below); it only grows, so that a wave that
  // reads it late sees a later tile's at worst
  const lds_int_ptr flag = (lds_int_ptr)(uintptr_t)(lds0 + S::FLAG);
  if (threadIdx.x == 0) *flag = 0;
  wait_lds();
  __builtin_amdgcn_s_barrier();
  int number = 0;
  // The ring: tile t is in stage t % NST; NST - 1 tiles are in flight ahead of the one being computed
  unsigned long long vis[NST - 1];                 // of the tiles in flight, the oldest first
  Unit cur = nxt;
  vis[0] = issue(0);
  if (NST > 2) {
    vis[NST - 2] = 0;
    if (left > 1) { advance(); vis[NST - 2] = issue(1); }
  }

  int stage = 0;
  while (left > 0) {
    // ---- a unit
    const int begin = cur.i, wave_row = row_base + wave * WROWS;
    Rows<D, RB> w;
    int wg_hi, wg_lo;                              // ... of the workgroup's rows
    int all_lo, all_hi;                            // keys that all of the wave's rows see: [all_lo, all_hi) as far as they exist
    {
      const Args a = arguments();
      const int g = a->g, last_row = cur.s.q_len * g - 1;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int R = min(wave_row + 16 * rb + l16, last_row), r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
        const uint16_t* qp = (const uint16_t*)a->q + cur.b * a->q_st[0] + hq * a->q_st[1] + r * a->q_st[2];
#pragma unroll
        for (int s2 = 0; s2 < NS; ++s2) w.q[rb][s2] = *reinterpret_cast<const bf16x8*>(qp + 32 * s2 + 8 * G);
        w.pos[rb] = cur.s.N - cur.s.q_len + r;
        w.neg_m[rb] = 0.f; w.thr[rb] = kNegBig; w.lsum[rb] = 0.f;
#pragma unroll
        for (int db = 0; db < NDB; ++db) w.o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      const int r0 = divide(min(wave_row, last_row), a->by_g), r1 = divide(min(wave_row + WROWS - 1, last_row), a->by_g);
      const int p0 = cur.s.N - cur.s.q_len;
      all_hi = a->causal ? p0 + r0 + 1 : 0x7fffffff;
      all_lo = a->window > 0 ? p0 + r1 - a->window + 1 : 0;
      wg_hi = a->causal ? cur.s.p0 + 1 : 0x7fffffff;
      wg_lo = a->window > 0 ? cur.s.p1 - a->window + 1 : 0;
    }
    if (NST > 2) wait_transfers();                 // the query rows: no wait for them is left to the loop
    bool taken = false;
    int i = begin;
    while (i < cur.T && left > 0) {
      // The tile has landed: transfers complete in order, and behind it at most those of one whole tile are in flight
      if (NST > 2 && left > 1) {
        asm volatile("" ::: "memory");
        wait_vmcnt<Slab<D>::IPT>();
        asm volatile("" ::: "memory");
      } else {
        wait_transfers();
      }
      // Rows at different positions and a tile that some see in part: the wave that moved a slab of V looks through it
      const int k0 = cur.s.tile(i) * kTK;
      const bool border = cur.s.p1 > cur.s.p0 && (k0 + kTK > wg_hi || (k0 < wg_lo && k0 + kTK > h.sinks));
      ++number;
      if (border && (NW == 4 || kind == 1)) {
        const unsigned at = lds_slab + S::VB + stage * S::STAGEB + 16 * fresh_lane();
        unsigned bad = 0;
#pragma unroll
        for (int t = 0; t < Slab<D>::IPT; ++t) bad |= nonfinite_bits((u32x4)*(lds_u32x4_ptr)(uintptr_t)(at + 1024 * t));
        if (__builtin_expect(__ballot(bad != 0) != 0, 0)) {
#pragma unroll
          for (int t = 0; t < Slab<D>::IPT; ++t) {
            const lds_u32x4_ptr p = (lds_u32x4_ptr)(uintptr_t)(at + 1024 * t);
            *p = __builtin_bit_cast(u32x4, finite_part(__builtin_bit_cast(s16x8, (u32x4)*p)));
          }
          *flag = number;
        }
      }
      wait_lds();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (border) taken |= uniform(*flag) >= number;
      const unsigned long long seen = vis[0];
      if (NST > 2) vis[0] = vis[NST - 2];
      if (left > NST - 1) {
        advance();
        vis[NST - 2] = issue(stage == 0 ? NST - 1 : stage - 1);
      }
      compute_tile<D, RB, NST>(h, w, kro + stage * S::STAGEB, vro + stage * S::STAGEB, k0, seen != ~0ull, k0 + kTK > all_hi,
                               k0 < all_lo && k0 + kTK > h.sinks, seen);
      ++i; --left;
      stage = stage == NST - 1 ? 0 : stage + 1;
    }

    // ---- this workgroup's share of the unit is done
    const Args a = arguments();
    const bool whole = begin == 0 && i == cur.T;
    const int g = a->g, last_row = cur.s.q_len * g - 1;
    const long long slot0 = slot * a->R;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float l = w.lsum[rb];
      const int R = wave_row + 16 * rb + l16;
      if (R > last_row) continue;
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const int r = divide(R, a->by_g), hq = cur.kvh * g + R - r * g;
        uint16_t* orow = (uint16_t*)a->out + cur.b * a->o_st[0] + hq * a->o_st[1] + r * a->o_st[2];
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          uint2 x;
          x.x = pack_bf16x2(w.o[rb][db][0] * inv, w.o[rb][db][1] * inv);
          x.y = pack_bf16x2(w.o[rb][db][2] * inv, w.o[rb][db][3] * inv);
          *reinterpret_cast<uint2*>(orow + 16 * db + 4 * G) = x;
        }
      } else {
#pragma unroll
        for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4*>(a->ws_o + (slot0 + R) * D + 16 * db + 4 * G) = w.o[rb][db];
        if (G == 0) { a->ws_ml[2 * (slot0 + R)] = w.thr[rb] == kNegBig ? kNegBig : -w.neg_m[rb]; a->ws_ml[2 * (slot0 + R) + 1] = l; }
      }
    }
    if (taken) put_back<uint16_t, D, kTK>(cur.s, cur.b, cur.kvh, begin, i, wave_row, WROWS, whole, a->ws_o + slot0 * D);
    if (FLAT) {
      slot = 2LL * blockIdx.x + 1;                 // the first unit's partial result goes to slot 0, the last's to 1
      if (left > 0) { cur.i = cur.T - 1; next_tile<kTK>(cur); }
    }
  }
}

// Merges the parts of a row that a row tile's workgroups left, in the order of the keys: GROUPS groups of D / 4 lanes per row
template <int D, int GROUPS>
__global__ __launch_bounds__(256) void paged_parts_merge_kernel(PagedArgs) {
  const Args a = arguments();
  constexpr int TPR = D / 4, RPB = 256 / (TPR * GROUPS);
  const int per_unit = (a->R + RPB - 1) / RPB, unit = blockIdx.x / (unsigned)per_unit;
  Part p;
  p.b = divide(unit, a->by_Hkv);
  const int b = p.b, kvh = unit - b * a->Hkv;
  int u0;
  find_part(-1, p, u0);
  const int R = (blockIdx.x - unit * per_unit) * RPB + threadIdx.x / (TPR * GROUPS), rt = divide(R, a->by_tile_rows);
  const Seen s = entry_seen<kTK>(a, p.len, p.q_len, rt);
  int n = 0;                                       // parts; of one, the workgroup has written the output
  if (R < s.q_len * a->g) {
    const int T = tiles_to_do(a, s, rt), per = (T + p.n - 1) / p.n;
    n = (T + per - 1) / per;
  }
  const RowSum sum = add_up<D, GROUPS>(a, 0, n - 1, [&](int k) { return (u0 + k * a->Hkv + kvh) * (long long)a->R + R; }, n > 1);
  if (n <= 1 || threadIdx.x / TPR % GROUPS != 0) return;
  const int d = threadIdx.x % TPR * 4;
  const f32x4 acc = sum.o;
  const float l = sum.l;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int r = divide(R, a->by_g), h = kvh * a->g + R - r * a->g;
  uint2 w2;
  w2.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  w2.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<uint2*>((uint16_t*)a->out + b * a->o_st[0] + h * a->o_st[1] + r * a->o_st[2] + d) = w2;
}

// ---- launch plan, from the parameters alone
// Rows of a workgroup and the sharing of the work by rows R per (sequence, K/V head) (us; lengths 500 to 8000, 8 sequences, heads of
// 128 unless stated):
//   up to 64: four waves of 16 rows, equal shares: 32 heads of 64 rows 130, in parts 145; 28 and 4 heads, 16 rows a head (R = 112) 40, in
//     parts 33
//   up to 256: four waves of 32 rows, in parts, whose row tiles find K and V in L2: R = 224 39 us, eight waves in shares 47; 32
//     sequences of 100 to 4000, R = 256, 129 and 168
//   more: eight waves of 32 rows, so that K and V come from L2 half as often: 2 x 2048 rows of 32 / 8 heads behind 4096 keys 321, four
//     waves 344; 8 x 512 rows over 4096 keys 257 and 271 (heads of 64: 188 and 190)
struct TilePlan { int rb, waves, flat, tile_rows, row_tiles, cuts; SharePlan shares; long long slots; };   // slots: parts at most

static TilePlan plan_tile(const sdllm_paged_attn_params& p, bool with_block) {
  const long long R = (long long)p.Hq / p.Hkv * p.K, units = (long long)p.B * p.Hkv;
  TilePlan pl{};
  pl.waves = R > 256 ? 8 : 4;
  pl.rb = R > 64 ? 2 : 1;
  const int rows = 16 * pl.rb * pl.waves, at_once = (pl.waves == 8 ? 1 : 2) * kNumCUs;
  pl.row_tiles = (int)((R + rows - 1) / rows);
  pl.tile_rows = rows;
  pl.flat = R <= 64;
  pl.cuts = 1;
  if (pl.flat) {
    pl.tile_rows = (int)R;
    pl.shares = plan_shares(p, with_block, pl.tile_rows, 1, kTK, at_once, 2);
    return pl;
  }
  const long long tiles = paged_most_tiles(p, with_block, rows, kTK), tiled = units * pl.row_tiles;
  const long long most = (1 << 20) / tiled;        // workgroups, and what the merge has to read, stay bounded
  const long long per = p.kv_splits > 0 ? (tiles + std::min<long long>(p.kv_splits, std::max(most, 1LL)) - 1) / std::min<long long>(p.kv_splits, std::max(most, 1LL)) : 2;
  if (tiles > per && p.B <= 2048 && units * R < (1 << 23) && (p.kv_splits > 0 || tiled < at_once)) {
    const long long workers = p.kv_splits > 0 ? 1 << 30 : at_once / pl.row_tiles;
    pl.shares = SharePlan{(int)workers, (int)per};
    pl.slots = std::min(units * ((tiles + per - 1) / per), workers);
    return pl;
  }
  while (pl.cuts < kNumXCDs && pl.cuts < pl.row_tiles && p.Hkv * pl.cuts % kNumXCDs != 0) pl.cuts *= 2;
  return pl;
}

size_t paged_tile_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  const TilePlan pl = plan_tile(p, with_block);
  if (pl.flat) return share_bytes(pl.shares, pl.tile_rows, p.D);
  return (size_t)pl.slots * (p.Hq / p.Hkv * p.K) * (p.D + 2) * sizeof(float);
}

template <int D, int RB, int NW, bool FLAT>
static hipError_t launch_tile(const PagedArgs& a, unsigned grid, hipStream_t stream, bool launch) {
  constexpr size_t bytes = TileShape<D, NW == 8 ? 3 : 2>::LDS;
  static LdsOptIn st;
  hipError_t e = ensure_lds_opt_in(reinterpret_cast<const void*>(&paged_tile_kernel<D, RB, NW, FLAT>), bytes, st);
  if (e != hipSuccess || !launch) return e;
  hipLaunchKernelGGL((paged_tile_kernel<D, RB, NW, FLAT>), dim3(grid), dim3(64 * NW), bytes, stream, a);
  return hipGetLastError();
}
template <int D>
static hipError_t launch_tile_d(const PagedArgs& a, const TilePlan& pl, unsigned grid, hipStream_t stream, bool launch = true) {
  if (pl.waves == 8) return launch_tile<D, 2, 8, false>(a, grid, stream, launch);
  return pl.flat ? launch_tile<D, 1, 4, true>(a, grid, stream, launch) : launch_tile<D, 2, 4, false>(a, grid, stream, launch);
}

hipError_t prepare_paged_tile() {
  hipError_t e = hipSuccess;
  for (int variant = 0; variant < 3; ++variant) {
    TilePlan pl{};
    pl.waves = variant == 2 ? 8 : 4; pl.flat = variant == 0;
    if (e == hipSuccess) e = launch_tile_d<64>(PagedArgs{}, pl, 0, nullptr, false);
    if (e == hipSuccess) e = launch_tile_d<128>(PagedArgs{}, pl, 0, nullptr, false);
  }
  return e;
}

hipError_t launch_paged_tile(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream) {
  const TilePlan pl = plan_tile(p, a.kb != nullptr);
  long long grid;
  set_shares(a, pl.shares, pl.tile_rows, pl.row_tiles, p.D, workspace);
  a.by_tile_rows = FastDiv(pl.tile_rows);
  a.cuts = pl.cuts;
  const long long units = (long long)p.B * p.Hkv;
  if (pl.flat) {
    grid = pl.shares.workers;
  } else if (pl.shares.min_tiles > 0) {
    a.ws_ml = a.ws_o + (size_t)pl.slots * a.R * p.D;
    grid = (pl.slots + kNumXCDs - 1) / kNumXCDs * kNumXCDs * pl.row_tiles;
  } else {
    grid = (units * pl.cuts + kNumXCDs - 1) / kNumXCDs * kNumXCDs * ((pl.row_tiles + pl.cuts - 1) / pl.cuts);
  }
  hipError_t e = p.D == 128 ? launch_tile_d<128>(a, pl, (unsigned)grid, stream) : launch_tile_d<64>(a, pl, (unsigned)grid, stream);
  if (e != hipSuccess || pl.shares.min_tiles == 0) return e;
  if (pl.flat) return launch_shares_merge(a, p.dtype, p.D, kTK, stream);
  const int all = 256 / (p.D / 4);
  // a workgroup per row for few rows of many parts (us, with the attention, a workgroup per row and not: 320 rows, 63 parts 17 and 22; 896
  // rows, 63 parts 28 and 31; 896 rows, 5 parts 16.5 and 15.3; 1792 rows, 32 parts 29.7 and 29.1)
  const bool alone = units * a.R <= kMergeAlone / 2 && pl.slots >= 16 * units;
  const dim3 grid_m((unsigned)(units * (alone ? a.R : (a.R + all - 1) / all)));
  if (p.D == 128) {
    if (alone) hipLaunchKernelGGL((paged_parts_merge_kernel<128, 8>), grid_m, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged_parts_merge_kernel<128, 1>), grid_m, dim3(256), 0, stream, a);
  } else {
    if (alone) hipLaunchKernelGGL((paged_parts_merge_kernel<64, 16>), grid_m, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((paged_parts_merge_kernel<64, 1>), grid_m, dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace sdllm
