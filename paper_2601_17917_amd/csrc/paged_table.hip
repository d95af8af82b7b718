// Block tables and slots of a paged K/V cache (sdllm_paged_extend) and the append of K/V rows into their slots
// (sdllm_paged_kv_append).
//
// Extend is prefix sums over the batch -- table entries of released sequences, which of them are pages, pages needed, pages granted
// so far -- and a fill of the tables and slots they decide.  It moves a few bytes per row, so what it costs is launches and dependent round trips: one workgroup
// does the scans and, where there are few rows, the fill behind them; many rows are filled by a second launch over the chip.
// Measured: 8 sequences of one row 2.0 us in the kernel; 64 of up to 2048 rows, a third of them new, 6.0 + 3.8 us.
#include "paged_common.h"

namespace sdllm {

struct ExtendArgs {
  int32_t* table; const int32_t* lens; const int32_t* new_lens; const uint8_t* do_append; const uint8_t* release;
  int32_t* free_pages; const int32_t* n_free; int32_t* lens_out; int32_t* n_free_out; int32_t* slots; int32_t* granted;
  int4* plan;                      // two launches: [B] of {length, rows granted, stack index of the first page, 0}
  int B, K, shift, max_pages, n_pages;
};

constexpr int kExtendOneLaunch = 16384;       // rows of the batch up to which the scanning workgroup fills them itself

// Inclusive sum over the workgroup of one value per thread; `total` receives the sum of all.  NT threads, 64-wide waves.
template <int NT>
__device__ __forceinline__ int block_scan(int v, int* wave_sums, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan(v);
  if (NT == 64) { total = __builtin_amdgcn_readlane(v, 63); return v; }
  __syncthreads();                            // the previous scan's sums are read
  if (lane == 63) wave_sums[wave] = v;
  __syncthreads();
  int before = 0; total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const int s = wave_sums[w];
    if (w < wave) before += s;
    total += s;
  }
  return v + before;
}

// Slot of row t of the n that sequence b takes on top of `len`, and the table entry if the row opens a page.  Its new pages are
// the stack entries top, top - 1, ...; entries of pages already held are read from the table, new ones from the stack, which
// does not change any more, so that no thread waits for another's store.
__device__ __forceinline__ void fill_slot(const ExtendArgs& a, int b, int len, int n, int top, int t) {
  int slot = -1;
  if (t < n) {
    const int mask = (1 << a.shift) - 1, pos = len + t, p = pos >> a.shift, held = (len + mask) >> a.shift;
    int32_t* entry = a.table + (long long)b * a.max_pages + p;
    const int page = p < held ? *entry : a.free_pages[top - (p - held)];
    if (p >= held && (pos & mask) == 0) *entry = page;
    if ((unsigned)page < (unsigned)a.n_pages) slot = (page << a.shift) + (pos & mask);
  }
  a.slots[(long long)b * a.K + t] = slot;
}

template <int NT, bool FILL>
__global__ __launch_bounds__(NT) void paged_extend_scan_kernel(ExtendArgs a) {
  __shared__ int wave_sums[16];
  __shared__ int s_first[NT], s_len[NT], s_n[NT];
  const int tid = threadIdx.x, mask = (1 << a.shift) - 1;
  const int cap = a.max_pages << a.shift;
  int avail = min(max(a.n_free[0], 0), a.n_pages);

  if (a.release != nullptr) {                  // pages that come back, in batch order
    constexpr int kReleaseLoads = NT == 64 ? 8 : 4;                   // table entries that a lane has in flight
    for (int b0 = 0; b0 < a.B; b0 += NT) {
      const int b = b0 + tid;
      int held = 0;
      if (b < a.B) {
        const int len = a.lens[b];                 // asked for at once with the flag
        held = a.release[b] != 0 ? (min(max(len, 0), cap) + mask) >> a.shift : 0;
      }
      // The entries of the chunk's released sequences, one row after the other; s_first: where a sequence's begin
      int all;
      const int upto = block_scan<NT>(held, wave_sums, all);
      s_first[tid] = upto - held;
      __syncthreads();
      auto sequence_of = [&](int e) {              // the last one that begins at e or before it: those without entries are in front of it
        int s = 0;
#pragma unroll
        for (int step = NT / 2; step > 0; step >>= 1)
          if (s_first[s + step] <= e) s += step;
        return s;
      };
      for (int e0 = 0; e0 < all; e0 += NT * kReleaseLoads) {
        const int e = e0 + tid * kReleaseLoads, n = min(kReleaseLoads, all - e);
        int id[kReleaseLoads];
        int s = 0, begin = 0, end = 0;             // entries of sequence s
#pragma unroll
        for (int u = 0; u < kReleaseLoads; ++u) {
          id[u] = -1;
          if (u >= n) continue;
          if (e + u >= end) {
            s = sequence_of(e + u);
            begin = s_first[s];
            end = s + 1 < NT ? s_first[s + 1] : all;
          }
          id[u] = a.table[(long long)(b0 + s) * a.max_pages + e + u - begin];
        }
        int pages = 0, got;                        // entries that are no pages stay behind
#pragma unroll
        for (int u = 0; u < kReleaseLoads; ++u) pages += (unsigned)id[u] < (unsigned)a.n_pages;
        int to = avail + block_scan<NT>(pages, wave_sums, got) - pages;
#pragma unroll
        for (int u = 0; u < kReleaseLoads; ++u)
          if ((unsigned)id[u] < (unsigned)a.n_pages && to < a.n_pages) a.free_pages[to++] = id[u];
        avail = min(avail + got, a.n_pages);
      }
    }
    __syncthreads();                           // pushed entries may be popped below
  }

  int needed = 0, taken = 0;                   // of all sequences before this chunk; pages that were granted
  for (int b0 = 0; b0 < a.B; b0 += NT) {
    const int b = b0 + tid;
    int len = 0, n = 0, need = 0;
    bool fits = false;
    if (b < a.B) {
      len = min(max(a.lens[b], 0), cap);
      if (a.release != nullptr && a.release[b] != 0) len = 0;
      n = a.new_lens != nullptr ? min(max(a.new_lens[b], 0), a.K) : a.K;
      if (a.do_append != nullptr && a.do_append[b] == 0) n = 0;
      fits = n <= cap - len;
      if (fits) need = ((len + n + mask) >> a.shift) - ((len + mask) >> a.shift);
    }
    int total;
    const int upto = needed + block_scan<NT>(need, wave_sums, total);       // at most B (K / 16 + 1)
    const bool ok = fits && (need == 0 || upto <= avail);
    const int first = avail - 1 - (upto - need);
    if (!ok) n = 0;
    if (b < a.B) {
      a.lens_out[b] = len + n;
      a.granted[b] = n;
    }
    int got;
    block_scan<NT>(ok ? need : 0, wave_sums, got);
    taken += got;
    needed += total;
    if constexpr (FILL) {
      __syncthreads();
      s_first[tid] = first; s_len[tid] = len; s_n[tid] = n;
      __syncthreads();
      const int seqs = min(NT, a.B - b0);
      for (int i = tid; i < seqs * a.K; i += NT) {
        const int s = i / a.K, t = i - s * a.K;
        fill_slot(a, b0 + s, s_len[s], s_n[s], s_first[s], t);
      }
    } else if (b < a.B) {
      a.plan[b] = int4{len, n, first, 0};
    }
  }
  if (tid == 0) a.n_free_out[0] = avail - taken;
}

constexpr int kFillRows = 1024;                // rows of a sequence that a workgroup fills

__global__ __launch_bounds__(256) void paged_extend_fill_kernel(ExtendArgs a, int parts) {
  const int b = blockIdx.x / (unsigned)parts, part = blockIdx.x - b * parts;
  const int4 pl = a.plan[b];
  const int t1 = min((part + 1) * kFillRows, a.K);
  for (int t = part * kFillRows + threadIdx.x; t < t1; t += 256) fill_slot(a, b, pl.x, pl.y, pl.z, t);
}

static bool extend_fills_itself(const sdllm_paged_extend_params& p) { return (long long)p.B * p.K <= kExtendOneLaunch; }

size_t paged_extend_workspace_bytes(const sdllm_paged_extend_params& p) {
  return extend_fills_itself(p) ? 0 : (size_t)p.B * sizeof(int4);
}

hipError_t launch_paged_extend(const sdllm_paged_extend_params& p, int32_t* table, const int32_t* lens, const int32_t* new_lens,
                               const uint8_t* do_append, const uint8_t* release, int32_t* free_pages, const int32_t* n_free,
                               int32_t* lens_out, int32_t* n_free_out, int32_t* slots, int32_t* granted, void* workspace,
                               hipStream_t stream) {
  ExtendArgs a;
  a.table = table; a.lens = lens; a.new_lens = new_lens; a.do_append = do_append; a.release = release;
  a.free_pages = free_pages; a.n_free = n_free; a.lens_out = lens_out; a.n_free_out = n_free_out; a.slots = slots; a.granted = granted;
  a.plan = (int4*)workspace;
  a.B = p.B; a.K = p.K; a.shift = __builtin_ctz(p.page_size); a.max_pages = p.max_pages; a.n_pages = p.n_pages;
  if (extend_fills_itself(p)) {
    if (p.B <= 64 && p.B * p.K <= 256) hipLaunchKernelGGL((paged_extend_scan_kernel<64, true>), dim3(1), dim3(64), 0, stream, a);
    else hipLaunchKernelGGL((paged_extend_scan_kernel<1024, true>), dim3(1), dim3(1024), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((paged_extend_scan_kernel<1024, false>), dim3(1), dim3(1024), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int parts = (p.K + kFillRows - 1) / kFillRows;
  hipLaunchKernelGGL(paged_extend_fill_kernel, dim3((unsigned)((long long)p.B * parts)), dim3(256), 0, stream, a, parts);
  return hipGetLastError();
}

// ---- append: one lane per 16 bytes, source contiguous; a row's slot is one (cached) load.  Slots outside the pool are skipped.
// Bound by HBM: 32 layers of 4 x 64 rows, 32 heads of 128, 268 MB in 47 us (5.7 TB/s).  The stores go past L2, which holds little of
// this for whoever reads it: through it 53 us, and 6.8 instead of 6.2 for 32 layers of 4 x 32 rows of 8 heads.  Scalar decoding of
// whole runs was no faster, eight accesses per lane were slower (75 us).
struct PagedAppendArgs {
  u32x4* kp; u32x4* vp; const u32x4* kb; const u32x4* vb; const int32_t* slots;
  long long pages_layer16, block_layer16;      // distances between layers, in 16-byte chunks
  long long chunks;                            // of one layer of one tensor
  FastDiv row16, K, Hkv;
  int shift, slots_total, parts;
};
constexpr int kPagedAppendUnroll = 4;

template <bool LARGE>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  const unsigned l = blockIdx.x / (unsigned)a.parts, part = blockIdx.x - l * (unsigned)a.parts;
  const u32x4* __restrict__ src = (blockIdx.y ? a.vb : a.kb) + (long long)l * a.block_layer16;
  u32x4* __restrict__ dst = (blockIdx.y ? a.vp : a.kp) + (long long)l * a.pages_layer16;
  const unsigned c0 = part * (256 * kPagedAppendUnroll) + threadIdx.x;
  u32x4 v[kPagedAppendUnroll]; int slot[kPagedAppendUnroll]; unsigned at[kPagedAppendUnroll];
#pragma unroll
  for (int u = 0; u < kPagedAppendUnroll; ++u) {
    const unsigned c = c0 + u * 256;
    slot[u] = -1;
    if (c >= a.chunks) continue;
    const unsigned row = a.row16.div(c), bh = a.K.div(row), t = row - bh * a.K.d, b = a.Hkv.div(bh), h = bh - b * a.Hkv.d;
    v[u] = LARGE ? __builtin_nontemporal_load(src + c) : src[c];
    slot[u] = a.slots[(long long)b * a.K.d + t];
    at[u] = (h << 16) | (c - row * a.row16.d);
  }
#pragma unroll
  for (int u = 0; u < kPagedAppendUnroll; ++u) {
    if ((unsigned)slot[u] >= (unsigned)a.slots_total) continue;
    const int page = slot[u] >> a.shift, r = slot[u] & ((1 << a.shift) - 1);
    const long long row = (((long long)page * a.Hkv.d + (at[u] >> 16)) << a.shift) + r;
    __builtin_nontemporal_store(v[u], dst + row * a.row16.d + (at[u] & 0xffff));
  }
}

hipError_t launch_paged_append(const sdllm_paged_append_params& p, void* k_pages, void* v_pages, const void* k_blocks,
                               const void* v_blocks, const int32_t* slots, hipStream_t stream) {
  const int elem = p.dtype == SDLLM_FP32 ? 4 : 2;
  PagedAppendArgs a;
  a.kp = (u32x4*)k_pages; a.vp = (u32x4*)v_pages; a.kb = (const u32x4*)k_blocks; a.vb = (const u32x4*)v_blocks; a.slots = slots;
  const int row16 = p.D * elem / 16;
  a.row16 = FastDiv(row16); a.K = FastDiv(p.K); a.Hkv = FastDiv(p.Hkv);
  a.shift = __builtin_ctz(p.page_size); a.slots_total = p.n_pages << a.shift;
  a.chunks = (long long)p.B * p.Hkv * p.K * row16;
  const long long dense_p = (long long)p.n_pages * p.page_size * p.Hkv * row16;
  a.pages_layer16 = p.pages_layer_stride ? p.pages_layer_stride * elem / 16 : dense_p;
  a.block_layer16 = p.block_layer_stride ? p.block_layer_stride * elem / 16 : a.chunks;
  a.parts = (int)((a.chunks + 256 * kPagedAppendUnroll - 1) / (256 * kPagedAppendUnroll));
  const long long blocks = (long long)p.n_layers * a.parts;
  // Loads past L2, too, of what it could not hold: 47 us instead of 48 for the 268 MB above, but 7.4 instead of 6.2 for 32 MB.
  if ((double)p.n_layers * a.chunks * 32 > 64e6) hipLaunchKernelGGL(paged_append_kernel<true>, dim3((unsigned)blocks, 2), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(paged_append_kernel<false>, dim3((unsigned)blocks, 2), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sdllm
