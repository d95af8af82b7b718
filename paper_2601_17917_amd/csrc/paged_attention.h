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
  unsigned page_bytes;                             // of one page, all heads
  int tile_rows, row_tiles;                        // query rows of a unit; units of a (sequence, K/V head)
  int workers, cuts, min_tiles;                    // how the key tiles are shared out (see the kernels)
  FastDiv by_g, by_row_tiles, by_Hkv, by_tile_rows;
  float scale_log2, thr8;                          // thr8: 8 in log2 units, as a difference of scores
};

// The kernels read their arguments where they use them: a fresh pointer that the compiler cannot see through, in a scope of its own,
// keeps what a unit's start and end need out of the registers of the loop between them.
typedef const __attribute__((address_space(4))) PagedArgs* Args;
__device__ __forceinline__ Args arguments() {
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}

__device__ __forceinline__ int divide(int n, const __attribute__((address_space(4))) FastDiv& by) {
  return (int)((__umulhi((unsigned)n, by.m) + (unsigned)n) >> by.s);
}
__device__ __forceinline__ long long quotient(long long n, long long d) {   // both >= 0; short where 32 bits do
  return ((unsigned long long)(n | d) >> 32) == 0 ? (unsigned)n / (unsigned)d : n / d;
}

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
  int last16, sink16;                              // 16 keys from k on are cached and seen if lo <= k <= last16, or k <= sink16
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : first + i - sink_tiles; }
};

__device__ __forceinline__ Seen seen_by(Args a, int n, int q_len, int r0, int r1, int TK) {
  Seen s;
  s.n = min(max(n, 0), a->max_kv);
  s.q_len = min(max(q_len, 0), a->K);
  s.N = s.n + (a->kb != nullptr ? s.q_len : 0);
  s.p0 = s.N - s.q_len + r0;
  s.p1 = s.N - s.q_len + min(r1, s.q_len - 1);
  s.hi = a->causal ? min(max(s.p1 + 1, 0), s.N) : s.N;
  s.lo = a->window > 0 ? min(max(s.p0 - a->window + 1, 0), s.hi) : 0;
  s.sink = min(a->sinks, s.lo);
  s.last16 = min(s.n, s.hi) - 16;
  s.first = s.lo / TK;
  s.sink16 = min(s.n, s.sink) - 16;
  s.sink_tiles = min((s.sink + TK - 1) / TK, s.first);
  s.tiles = s.sink_tiles + (s.hi + TK - 1) / TK - s.first;       // lo < hi unless both are 0: then none
  return s;
}

// Keys visible to row r of the tile: [lo, hi) and below sinks
__device__ __forceinline__ void row_range(Args a, const Seen& s, int r, int& lo, int& hi) {
  const int p = s.N - s.q_len + r;
  hi = a->causal ? min(max(p + 1, 0), s.N) : s.N;
  lo = a->window > 0 ? max(p - a->window + 1, 0) : 0;
}

// The lane, made anew: what a slower path derives from it is not kept in registers over the loop
__device__ __forceinline__ int fresh_lane() {
  int x = threadIdx.x;
  asm volatile("" : "+v"(x));
  return x & 63;
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

// The call's units: row tile rt of sequence b (entry e = b row_tiles + rt), once for each K/V head.  What an entry sees:
template <int TK>
__device__ __forceinline__ Seen entry_seen(Args a, int n, int q_len, int rt) {
  return seen_by(a, n, q_len, divide(rt * a->tile_rows, a->by_g), divide((rt + 1) * a->tile_rows - 1, a->by_g), TK);
}
__device__ __forceinline__ int tiles_to_do(Args a, const Seen& s, int rt) {
  // rows that see nothing are a tile of their own: they are zero
  return rt * a->tile_rows < s.q_len * a->g ? max(s.tiles, 1) : 0;
}
// Key tiles of entries e0 .. e0 + 63, one per lane, and their sums up to the lane (below 2^31 where keys are shared out, plan_shares)
struct Entries { int n, q_len, tiles, upto; };
template <int TK>
__device__ __forceinline__ Entries entries(Args a, int e0) {
  Entries x{0, 0, 0, 0};
  const int e = e0 + (int)(threadIdx.x & 63);
  if (e < a->B * a->row_tiles) {
    const int b = divide(e, a->by_row_tiles), rt = e - b * a->row_tiles;
    x.n = a->lens[b];
    x.q_len = a->q_lens ? a->q_lens[b] : a->K;
    x.tiles = tiles_to_do(a, entry_seen<TK>(a, x.n, x.q_len, rt), rt);
  }
  x.upto = wave_scan(x.tiles);
  return x;
}
__device__ __forceinline__ int read_lane(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ long long tiles_per_worker(Args a, long long total) {
  const long long n = quotient(total + a->workers - 1, a->workers);
  return n > a->min_tiles ? n : a->min_tiles;
}

// A unit being walked; everything uniform
struct Unit {
  int e, b, rt, kvh, i, T;                         // tile i of T
  Seen s;
};

template <int TK>
__device__ __forceinline__ void open_unit(Unit& u, int e, int kvh, int i, int n, int q_len) {
  const Args a = arguments();
  u.e = e; u.b = divide(e, a->by_row_tiles); u.rt = e - u.b * a->row_tiles; u.kvh = kvh; u.i = i;
  u.s = entry_seen<TK>(a, n, q_len, u.rt);
  u.T = tiles_to_do(a, u.s, u.rt);
}
template <int TK>
__device__ __forceinline__ void open_unit(Unit& u, int e, int kvh, int i) {
  const Args a = arguments();
  const const_i32_ptr lens = (const_i32_ptr)(uintptr_t)a->lens, q_lens = (const_i32_ptr)(uintptr_t)a->q_lens;
  const int b = divide(e, a->by_row_tiles);
  open_unit<TK>(u, e, kvh, i, lens[b], a->q_lens ? q_lens[b] : a->K);
}

// The unit and tile that the share of worker w begins with; returns the tiles of the share (0: none)
template <int TK>
__device__ __forceinline__ int open_share(int w, Unit& u) {
  const Args a = arguments();
  const int E = a->B * a->row_tiles;
  Entries x = entries<TK>(a, 0);
  int chunk = read_lane(x.upto, 63);
  long long total = chunk;
  for (int e0 = 64; e0 < E; e0 += 64) total += read_lane(entries<TK>(a, e0).upto, 63);
  total *= a->Hkv;
  const long long per = tiles_per_worker(a, total), f = w * per;
  if (f >= total) return 0;
  long long rest = f;                              // tiles in front of it, from entry e0 on
  int e0 = 0;
  while (rest >= (long long)chunk * a->Hkv) {
    rest -= (long long)chunk * a->Hkv;
    e0 += 64;
    x = entries<TK>(a, e0);
    chunk = read_lane(x.upto, 63);
  }
  const int l = __builtin_ctzll(__ballot((long long)x.upto * a->Hkv > rest));
  const int t = read_lane(x.tiles, l);
  rest -= (long long)(read_lane(x.upto, l) - t) * a->Hkv;
  const int kvh = (int)quotient(rest, t);
  open_unit<TK>(u, e0 + l, kvh, (int)(rest - (long long)kvh * t), read_lane(x.n, l), read_lane(x.q_len, l));
  return (int)(per < total - f ? per : total - f);
}
template <int TK>
__device__ __forceinline__ void next_tile(Unit& u) {
  if (++u.i < u.T) return;
  const Args a = arguments();
  if (u.kvh + 1 < a->Hkv) { ++u.kvh; u.i = 0; return; }
  int e = u.e;
  do { open_unit<TK>(u, ++e, 0, 0); } while (u.T == 0 && e + 1 < a->B * a->row_tiles);
}

// What the loop over tiles needs of the arguments
struct Hot {
  const unsigned char* kp; const unsigned char* vp;
  unsigned page_bytes; int n_pages, shift, last_page, window, sinks;
  float scale_log2, thr8;
};
__device__ __forceinline__ Hot hot_arguments() {
  const Args a = arguments();
  Hot h;
  h.kp = (const unsigned char*)a->kp; h.vp = (const unsigned char*)a->vp;
  h.page_bytes = a->page_bytes; h.n_pages = a->n_pages; h.shift = a->shift; h.last_page = a->max_pages - 1; h.sinks = a->sinks; h.window = a->window;
  h.scale_log2 = a->scale_log2; h.thr8 = a->thr8;
  // each in a register of its own, not a part of the tuples they were loaded in
  asm volatile("" : "+s"(h.kp), "+s"(h.vp), "+s"(h.page_bytes), "+s"(h.n_pages), "+s"(h.shift), "+s"(h.last_page), "+s"(h.sinks), "+s"(h.window),
               "+s"(h.scale_log2), "+s"(h.thr8));
  return h;
}
// The 64 entries of a sequence's block table around the current tile, one per lane: a tile's page ids are lane reads, and memory is
// only asked again 64 pages further on.  (A scalar load per tile would make every LDS wait behind it a wait for it, too.)
struct Pages {
  const int32_t* row;                              // of the sequence
  int block, id;                                   // entry 64 block + lane
  unsigned long long valid;                        // which of them are pages of the pool
  __device__ __forceinline__ void open(int b) {
    const Args a = arguments();
    row = a->table + (long long)b * a->max_pages;
    block = -1;
  }
  __device__ __forceinline__ void seek(const Hot& h, int k) {          // to the tile at key k
    const int want = k >> (h.shift + 6);
    if (want == block) return;
    block = want;
    id = row[min(64 * want + fresh_lane(), h.last_page)];   // entries behind the table's end repeat the last one
    valid = __ballot((unsigned)id < (unsigned)h.n_pages);
  }
  // keys [begin, valid_until) are in valid pages of these entries, one after the other
  __device__ __forceinline__ int begin(const Hot& h) const { return block << (h.shift + 6); }
  __device__ __forceinline__ int valid_until(const Hot& h) const {
    return begin(h) + ((~valid == 0 ? 64 : __builtin_ctzll(~valid)) << h.shift);
  }
  __device__ __forceinline__ int of(const Hot& h, int k) const { return __builtin_amdgcn_readlane(id, (k >> h.shift) & 63); }
  __device__ __forceinline__ bool ok(const Hot& h, int k) const { return (valid >> ((k >> h.shift) & 63)) & 1; }
  // all pages of the TK keys from k on (a multiple of TK)
  template <int TK> __device__ __forceinline__ bool all_ok(const Hot& h, int k) const {
    const int n = TK >> h.shift;                   // pages of the tile, if more than one
    const unsigned long long want = n > 1 ? (1ull << n) - 1 : 1;
    return ((valid >> ((k >> h.shift) & 63)) & want) == want;
  }
};
// Opens a unit whose number is known from the start: its lengths and its first table entries travel together
template <int TK>
__device__ __forceinline__ void open_whole_unit(Unit& u, Pages& pages, const Hot& h, int unit) {
  const Args a = arguments();
  const const_i32_ptr lens = (const_i32_ptr)(uintptr_t)a->lens, q_lens = (const_i32_ptr)(uintptr_t)a->q_lens;
  const int e = divide(unit, a->by_Hkv), b = divide(e, a->by_row_tiles);
  const int n = lens[b], q_len = a->q_lens ? q_lens[b] : a->K;
  pages.open(b);
  pages.seek(h, 0);
  open_unit<TK>(u, e, unit - e * a->Hkv, 0, n, q_len);
}
// Byte offset in kp / vp of row k of K/V head kvh, which lies in page id
__device__ __forceinline__ unsigned long long row_offset(const Hot& h, int id, int kvh, int k, int row_bytes) {
  return (unsigned long long)(unsigned)id * h.page_bytes + (unsigned)(((kvh << h.shift) + (k & ((1 << h.shift) - 1))) * row_bytes);
}

// ---- K/V rows global -> LDS, in slabs of 16 rows.  LDS rows are unpadded; 16-byte chunk c of row r lies at c ^ f(r), f_K(r) = (r / R256)
// mod CPR, f_V(r) = 2 ((r / R256) mod (CPR / 2)), which keeps the operand reads free of bank conflicts (as in the dense kernel).
template <int D> struct Slab {
  static constexpr int CPR = D / 8;                // chunks per row
  static constexpr int RPI = 64 / CPR;             // rows per wave-wide transfer
  static constexpr int IPT = 16 / RPI;             // transfers per slab
  static constexpr int R256 = 16 / CPR;            // rows per 256 bytes
  static constexpr int ROWB = D * 2, BYTES = 16 * ROWB;
  // where chunk c of row r lies in its LDS row (and which chunk lies at c)
  __host__ __device__ static constexpr int at(bool v, int r, int c) { return c ^ (v ? 2 * ((r / R256) % (CPR / 2)) : (r / R256) % CPR); }
  // byte within the source of the lane's chunk of transfer 0, and the bits of it that transfer j flips (less j KiB, dma_slab)
  __device__ static unsigned lane_offset(bool v) {
    const int lane = fresh_lane(), r = lane / CPR, c = lane % CPR;
    return r * ROWB + (at(v, r, c) << 4);
  }
  // The same for rows `stride` bytes apart, transfer j.  The hardware adds it to a scalar address as an unsigned number of 32 bits, so it
  // must not be negative: transfer j begins with row RPI j, which is j KiB in or more if rows do not overlap (RPI ROWB = 1 KiB).
  __host__ __device__ static constexpr unsigned strided_offset(bool v, int lane, int j, unsigned stride) {
    const int r = RPI * j + lane / CPR;
    return r * stride + (at(v, r, lane % CPR) << 4) - 1024 * j;
  }
  __host__ __device__ static constexpr bool strided(long long stride) { return stride >= ROWB && stride < (1 << 27); }
  __device__ static constexpr unsigned flips(bool v, int j) { return v ? (D == 128 ? 128 * (j & 1) : 0) : 64 * j; }
  __device__ static __forceinline__ void offsets(bool v, unsigned (&off)[4]) {
    const unsigned g = lane_offset(v);
#pragma unroll
    for (int j = 0; j < 4; ++j) off[j] = g ^ flips(v, j);
  }
};

// Whole slab from consecutive rows; V: which tensor's order.  (The offsets are made here: kept over a loop they cost registers.)
template <int D, bool ONCE, bool V>
__device__ __forceinline__ void move_slab(unsigned lds, const unsigned char* src) {
  unsigned off[4];
  Slab<D>::offsets(V, off);
  dma_slab<Slab<D>::IPT, ONCE>(lds, uniform_ptr(src), off);
}

// Whole slab from 16 rows `stride` bytes apart (a block's rows as a projection leaves them)
template <int D, bool ONCE, bool V>
__device__ __forceinline__ void move_strided(unsigned lds, const unsigned char* src, unsigned stride) {
  using S = Slab<D>;
  const int lane = fresh_lane();
  unsigned off[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) off[j] = S::strided_offset(V, lane, j < S::IPT ? j : 0, stride);
  dma_slab<S::IPT, ONCE>(lds, uniform_ptr(src), off);
}
// The block's rows of a (sequence, K/V head)
template <int D> struct BlockRows {
  const unsigned char *k, *v;                      // of row 0
  unsigned k_stride, v_stride;                     // bytes between rows; 0: no block, or rows that only move_rows can address
  __device__ __forceinline__ void open(int b, int kvh) {
    const Args a = arguments();
    k_stride = v_stride = 0;
    k = v = nullptr;
    if (a->kb == nullptr || !Slab<D>::strided(2 * a->kb_st[2]) || !Slab<D>::strided(2 * a->vb_st[2])) return;
    k = (const unsigned char*)a->kb + 2 * (b * a->kb_st[0] + kvh * a->kb_st[1]);
    v = (const unsigned char*)a->vb + 2 * (b * a->vb_st[0] + kvh * a->vb_st[1]);
    k_stride = (unsigned)(2 * a->kb_st[2]); v_stride = (unsigned)(2 * a->vb_st[2]);
  }
};

// Which of the TK keys from k on (a multiple of 16) some query row sees and has a page: bit r: key k + r
template <int TK>
__device__ __forceinline__ unsigned long long seen_keys(const Hot& h, const Seen& s, const Pages& p, int k) {
  const int lane = fresh_lane(), key = k + lane;
  bool page = false;
#pragma unroll
  for (int j = 0; j < TK / 16; ++j) page |= (lane >> 4) == j && p.ok(h, k + 16 * j);
  return __ballot((lane < TK) & (key < s.hi) & ((key >= s.lo) | (key < s.sink)) & ((key >= s.n) | page));
}

// Rows of a slab from wherever they lie, zeros for those whose bit is not set.  page_row: address of key k in its page.
template <int D, bool ONCE, bool V>
__device__ __forceinline__ void move_rows(const Seen& s, int b, int kvh, int k, unsigned bits, const unsigned char* page_row, unsigned lds,
                                          unsigned char* lds_ptr) {
  using S = Slab<D>;
  const int lane = fresh_lane(), c = lane % S::CPR;
#pragma unroll
  for (int t = 0; t < S::IPT; ++t) *reinterpret_cast<u32x4*>(lds_ptr + 1024 * t + 16 * lane) = u32x4{0, 0, 0, 0};
  wait_lds();
  if (bits == 0) return;
  const Args a = arguments();
  const unsigned char* block = (const unsigned char*)(V ? a->vb : a->kb);
  const long long st = V ? a->vb_st[2] : a->kb_st[2];
  if (block != nullptr) block += 2 * (b * (V ? a->vb_st[0] : a->kb_st[0]) + kvh * (V ? a->vb_st[1] : a->kb_st[1]) + (k - s.n) * st);
#pragma unroll 1
  for (int t = 0; t < S::IPT; ++t) {
    const int r = S::RPI * t + lane / S::CPR;
    const int at = S::at(V, r, c) << 4;
    if ((bits >> r) & 1) dma16_vaddr<ONCE>(lds + 1024 * t, (k + r < s.n ? page_row + r * S::ROWB : block + 2 * r * st) + at);
  }
}

// Scores of hidden keys become -inf.  Score [kb][e] of a lane is key k0 + 16 kb + 4 G + e of its row, which sees keys [lo, hi) and
// those below sinks; bit 16 kb + 4 G + e of vis: the key exists.  Border by border: most tiles that have one have one kind.
template <int KB>
__device__ __forceinline__ void hide(f32x4 (&z)[KB], int k0, int lo, int hi, int sinks, unsigned long long vis, bool some_missing,
                                     bool above, bool below) {
  const int G4 = (fresh_lane() >> 4) * 4;
  if (some_missing) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const unsigned bits = (unsigned)(vis >> (16 * kb)) >> G4;
#pragma unroll
      for (int e = 0; e < 4; ++e) z[kb][e] = (bits >> e) & 1 ? z[kb][e] : -INFINITY;
    }
  }
  if (above) {
    const int t = hi - k0 - G4;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[kb][e] = 16 * kb + e < t ? z[kb][e] : -INFINITY;
  }
  if (below) {
    const int t = lo - k0 - G4, u = sinks - k0 - G4;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[kb][e] = ((16 * kb + e >= t) | (16 * kb + e < u)) ? z[kb][e] : -INFINITY;
  }
}

// ---- Values that are not finite, in a tile whose keys some rows see and others do not: a weight of 0 times such a value would be NaN
// in the rows that do not see it.  The kernels look for them in such tiles only, take them as 0 there, and have them added to the rows
// that see one at the end (put_back).
// Bits 15 and 31 of the result: one of the low / high bf16 of x has an exponent of all ones.
__device__ __forceinline__ unsigned nonfinite_bits(const u32x4& x) {
  unsigned bad = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) bad |= (x[w] & 0x7f807f80u) + 0x00800080u;
  return bad & 0x80008000u;
}
__device__ __forceinline__ s16x8 finite_part(const s16x8& v) {
  u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const unsigned bad = ((x[w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    x[w] &= ~(bad - (bad >> 15));                  // 0x7fff in the halves to clear: +0 or -0
  }
  return __builtin_bit_cast(s16x8, x);
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((unsigned)x << 16); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }

// Adds what was taken out of a unit's tiles [i0, i1) to those of the rows R0 .. R0 + count - 1 that see it, in the output or in a partial result
// (that of row 0: part_o), where the caller has written the rest: a weight is positive, so that its product with such a value is the
// value.  Only tiles that some row sees in part are looked through, whatever the length: 2 x 2048 causal rows of 32 / 8 heads behind 6000 keys,
// an infinity in each head, 0.34 -> 0.39 ms.  (To add what another tile's products have added already changes nothing.)
template <typename T, int D, int TK>
__device__ __forceinline__ void put_back(const Seen& s, int b, int kvh, int i0, int i1, int R0, int count, bool whole, float* part_o) {
  const Args a = arguments();
  const int lane = threadIdx.x & 63, rows = min(R0 + count, s.q_len * a->g);
  if (R0 >= rows) return;
  const int32_t* table = a->table + (long long)b * a->max_pages;
  wait_transfers();                                // what the caller has written is in front of what is read here
  wait_lds();
#pragma unroll 1
  for (int first = i0; first < i1; first += 64) {
    bool in_part = false;                          // a lane per tile: beyond what all rows see, or with a page that is not there
    if (first + lane < i1) {
      const int k0 = s.tile(first + lane) * TK;
      in_part = k0 + TK > (a->causal ? s.p0 + 1 : s.N) || (a->window > 0 && k0 < s.p1 - a->window + 1 && k0 + TK > a->sinks);
      for (int e = k0 >> a->shift; e <= (min(k0 + TK, s.n) - 1) >> a->shift; ++e) in_part |= (unsigned)table[e] >= (unsigned)a->n_pages;
    }
#pragma unroll 1
    for (unsigned long long tiles = __ballot(in_part); tiles != 0; tiles &= tiles - 1) {
      const int key = s.tile(first + __builtin_ctzll(tiles)) * TK + lane;
      // its rows of V, a lane per key
      const T* v = nullptr;
      bool there = lane < TK && key < s.N;
      if (there) {
        if (key < s.n) {
          const int page = table[key >> a->shift];
          there = (unsigned)page < (unsigned)a->n_pages;
          v = (const T*)a->vp + ((((long long)page * a->Hkv + kvh) << a->shift) + (key & ((1 << a->shift) - 1))) * D;
        } else {
          v = (const T*)a->vb + b * a->vb_st[0] + kvh * a->vb_st[1] + (key - s.n) * a->vb_st[2];
        }
      }
      auto value = [&](int j, int u) {             // of key j, a lane per column
        return to_float(((const T*)(uintptr_t)__shfl((unsigned long long)(uintptr_t)v, j))[lane + 64 * u]);
      };
      unsigned long long bad = 0;                  // keys with a value that is not finite
#pragma unroll 1
      for (unsigned long long keys = __ballot(there); keys != 0; keys &= keys - 1) {
        const int j = __builtin_ctzll(keys);
        bool finite = true;
#pragma unroll
        for (int u = 0; u < D / 64; ++u) finite &= __builtin_isfinite(value(j, u));
        if (__ballot(!finite) != 0) bad |= 1ull << j;
      }
      if (bad == 0) continue;
#pragma unroll 1
      for (int R = R0; R < rows; ++R) {
        const int r = divide(R, a->by_g), h = kvh * a->g + R - r * a->g;
        int lo, hi;
        row_range(a, s, r, lo, hi);
        float sum[D / 64] = {};
#pragma unroll 1
        for (unsigned long long keys = __ballot((key < hi) & ((key >= lo) | (key < a->sinks))) & bad; keys != 0; keys &= keys - 1) {
          const int j = __builtin_ctzll(keys);
#pragma unroll
          for (int u = 0; u < D / 64; ++u) {
            const float x = value(j, u);
            sum[u] += __builtin_isfinite(x) ? 0.f : x;
          }
        }
#pragma unroll
        for (int u = 0; u < D / 64; ++u) {
          if (__builtin_isfinite(sum[u])) continue;
          const int d = lane + 64 * u;
          if (whole) {
            T* out = (T*)a->out + b * a->o_st[0] + h * a->o_st[1] + r * a->o_st[2] + d;
            put(out, to_float(*out) + sum[u]);
          } else {
            part_o[(long long)R * D + d] += sum[u];
          }
        }
      }
    }
  }
}

// Output of `rows` query rows (from R0 on) of a unit that the waves of a workgroup walked together: n partial results in LDS, wave_o
// floats apart (rows of D) and wave_ml floats apart (reference, sum)
template <typename T, int D, int THREADS>
__device__ __forceinline__ void merge_waves(const Unit& u, int R0, int rows, int n, const float* o_s, int wave_o, const float* ml_s, int wave_ml) {
  const Args a = arguments();
  constexpr int TPR = D / 4;
  for (int x = threadIdx.x; x < rows * TPR; x += THREADS) {
    const int row = x / TPR, d = x % TPR * 4, R = R0 + row;
    if (R >= u.s.q_len * a->g) break;
    float M = kNegBig, l = 0.f;
    for (int k = 0; k < n; ++k) M = fmaxf(M, ml_s[k * wave_ml + 2 * row]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < n; ++k) {
      const float c = exp2_fast((ml_s[k * wave_ml + 2 * row] - M) * a->scale_log2);
      acc += *reinterpret_cast<const f32x4*>(o_s + k * wave_o + row * D + d) * c;
      l += ml_s[k * wave_ml + 2 * row + 1] * c;
    }
    acc *= l == 0.f ? 0.f : 1.0f / l;
    const int r = divide(R, a->by_g), h = u.kvh * a->g + R - r * a->g;
    T* out = (T*)a->out + u.b * a->o_st[0] + h * a->o_st[1] + r * a->o_st[2] + d;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(out) = acc;
    } else {
      uint2 w;
      w.x = pack_bf16x2(acc[0], acc[1]);
      w.y = pack_bf16x2(acc[2], acc[3]);
      *reinterpret_cast<uint2*>(out) = w;
    }
  }
}

// Adds up the partial results first .. last of a row (slot(k): where the k-th lies, in rows), in groups of D / 4 lanes that take every
// GROUPS-th each; then group 0 adds up the groups, in order.  All threads of the workgroup call it; the sum is group 0's.
struct RowSum { f32x4 o; float m, l; };
template <int D, int GROUPS, typename Slot>
__device__ __forceinline__ RowSum add_up(Args a, int first, int last, Slot&& slot, bool exists) {
  constexpr int TPR = D / 4;
  const int grp = threadIdx.x / TPR % GROUPS, d = threadIdx.x % TPR * 4;
  RowSum s{f32x4{0.f, 0.f, 0.f, 0.f}, kNegBig, 0.f};
  auto add = [&](float mk, float lk, const f32x4& ov) {
    const float up = fmaxf(s.m, mk), c0 = exp2_fast((s.m - up) * a->scale_log2), c1 = exp2_fast((mk - up) * a->scale_log2);
    s.o = s.o * c0 + ov * c1;
    s.l = s.l * c0 + lk * c1;
    s.m = up;
  };
  if (exists) {
    int k = first + grp;
    for (; k + 3 * GROUPS <= last; k += 4 * GROUPS) {          // four partial results' loads together
      f32x4 ov[4]; float mk[4], lk[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const long long at = slot(k + u * GROUPS);
        ov[u] = *reinterpret_cast<const f32x4*>(a->ws_o + at * D + d);
        mk[u] = a->ws_ml[2 * at]; lk[u] = a->ws_ml[2 * at + 1];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) add(mk[u], lk[u], ov[u]);
    }
    for (; k <= last; k += GROUPS) {
      const long long at = slot(k);
      add(a->ws_ml[2 * at], a->ws_ml[2 * at + 1], *reinterpret_cast<const f32x4*>(a->ws_o + at * D + d));
    }
  }
  if constexpr (GROUPS > 1) {
    __shared__ f32x4 o_s[256];
    __shared__ float m_s[256 / TPR], l_s[256 / TPR];
    const int row0 = threadIdx.x / TPR - grp;                  // group 0 of the row
    o_s[threadIdx.x] = s.o;
    if (d == 0) { m_s[row0 + grp] = s.m; l_s[row0 + grp] = s.l; }
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int k = 1; k < GROUPS; ++k) add(m_s[row0 + k], l_s[row0 + k], o_s[(row0 + k) * TPR + d / 4]);
    }
  }
  return s;
}
// Rows up to which each has a workgroup of its own for that: that many are on the chip at once, and what counts is the way through a
// row's shares.  With more rows it is the number of workgroups.  (us with the attention itself, alone and in workgroups of eight rows, heads
// of 128: 32 rows, one sequence of 32768 keys 31 and 46; 2048 rows, 8 of 4096 36 and 35; 4096 rows, 16 of 4096 58 and 54; 8192 rows, 32 of
// 4096 102 and 93.)
constexpr int kMergeAlone = 8 * kNumCUs;

// Kernels: bf16 by query rows per (sequence, K/V head), up to 32 (stream) and more (tile); fp32
size_t paged_stream_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block);
hipError_t launch_paged_stream(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream);
size_t paged_tile_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block);
hipError_t launch_paged_tile(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream);
size_t paged_f32_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block);
hipError_t launch_paged_f32(const sdllm_paged_attn_params& p, PagedArgs& a, void* workspace, hipStream_t stream);

// Most key tiles of TK that a unit of `rows` query rows can have
long long paged_most_tiles(const sdllm_paged_attn_params& p, bool with_block, long long rows, int TK);
// Units in equal shares: workers, tiles of a share at least, 0: a worker per unit and no merge
struct SharePlan { int workers, min_tiles; };
SharePlan plan_shares(const sdllm_paged_attn_params& p, bool with_block, int tile_rows, int row_tiles, int TK, int at_once, int min_tiles);
size_t share_bytes(const SharePlan& pl, int tile_rows, int D);
void set_shares(PagedArgs& a, const SharePlan& pl, int tile_rows, int row_tiles, int D, void* workspace);
hipError_t launch_shares_merge(const PagedArgs& a, int dtype, int D, int TK, hipStream_t stream);

}  // namespace sdllm
