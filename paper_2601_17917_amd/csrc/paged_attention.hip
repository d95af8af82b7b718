// sdllm_paged_attention: dispatch, the plan by equal shares that its kernels have in common, and the merge of the shares.
#include "paged_attention.h"
#include <cmath>

namespace sdllm {

// Merges the shares of every output row that several workers walked, in the order of the tiles: GROUPS groups of D / 4 lanes per row
template <typename T, int D, int TK, int GROUPS>
__global__ __launch_bounds__(256) void shares_merge_kernel(PagedArgs) {
  const Args a = arguments();
  constexpr int TPR = D / 4, RPW = 256 / (TPR * GROUPS);
  const int grp = threadIdx.x / TPR % GROUPS, d = threadIdx.x % TPR * 4;
  // the rows of a workgroup: of one (sequence, K/V head, row tile)
  const int per_tile = (a->tile_rows + RPW - 1) / RPW;
  const unsigned tile = blockIdx.x / (unsigned)per_tile;
  const int e = divide(tile, a->by_Hkv), kvh = tile - e * a->Hkv, b = divide(e, a->by_row_tiles), rt = e - b * a->row_tiles;
  const int row = (blockIdx.x - tile * per_tile) * RPW + threadIdx.x / (TPR * GROUPS), R = rt * a->tile_rows + row;
  // where the unit's tiles lie among the call's
  long long total = 0, start = 0;
  int n = 0;
  for (int e0 = 0; e0 < a->B * a->row_tiles; e0 += 64) {
    const Entries x = entries<TK>(a, e0);
    if (e >= e0 && e < e0 + 64) {
      n = read_lane(x.tiles, e - e0);
      start = (total + read_lane(x.upto, e - e0) - n) * a->Hkv + (long long)kvh * n;
    }
    total += read_lane(x.upto, 63);
  }
  total *= a->Hkv;
  if (n == 0) return;
  const long long per = tiles_per_worker(a, total);
  const int w0 = (int)quotient(start, per), w1 = (int)quotient(start + n - 1, per);
  if (w0 == w1) return;                            // written by its worker
  const int q_len = min(max(a->q_lens ? a->q_lens[b] : a->K, 0), a->K);
  const bool exists = row < a->tile_rows && R < q_len * a->g;
  // a unit is its worker's first one unless the worker began before it
  const RowSum sum = add_up<D, GROUPS>(a, w0, w1, [&](int w) { return ((long long)w * 2 + (start > w * per ? 1 : 0)) * a->tile_rows + row; }, exists);
  if (grp != 0 || !exists) return;
  const f32x4 acc = sum.o;
  const float l = sum.l;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int r = divide(R, a->by_g), h = kvh * a->g + R - r * a->g;
  T* out = (T*)a->out + b * a->o_st[0] + h * a->o_st[1] + r * a->o_st[2] + d;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(out) = acc * inv;
  } else {
    uint2 w2;
    w2.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    w2.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
    *reinterpret_cast<uint2*>(out) = w2;
  }
}

template <typename T, int D, int TK>
static void launch_merge(const PagedArgs& a, hipStream_t stream) {
  constexpr int all = 256 / (D / 4);
  const long long units = (long long)a.B * a.Hkv * a.row_tiles;
  if (units * a.tile_rows <= kMergeAlone) {
    hipLaunchKernelGGL((shares_merge_kernel<T, D, TK, all>), dim3((unsigned)(units * a.tile_rows)), dim3(256), 0, stream, a);
  } else {
    const int per_tile = (a.tile_rows + all - 1) / all;
    hipLaunchKernelGGL((shares_merge_kernel<T, D, TK, 1>), dim3((unsigned)(units * per_tile)), dim3(256), 0, stream, a);
  }
}

hipError_t launch_shares_merge(const PagedArgs& a, int dtype, int D, int TK, hipStream_t stream) {
  if (dtype == SDLLM_FP32) {
    if (D == 128) launch_merge<float, 128, 16>(a, stream);
    else launch_merge<float, 64, 16>(a, stream);
  } else if (D == 64) {
    launch_merge<uint16_t, 64, 64>(a, stream);
  } else if (TK == 32) {
    launch_merge<uint16_t, 128, 32>(a, stream);
  } else {
    launch_merge<uint16_t, 128, 64>(a, stream);
  }
  return hipGetLastError();
}

long long paged_most_tiles(const sdllm_paged_attn_params& p, bool with_block, long long rows, int TK) {
  const long long N = p.max_kv_len + (with_block ? p.K : 0), g = p.Hq / p.Hkv;
  long long tiles = (N + TK - 1) / TK;
  if (p.window > 0) {
    const long long span = (rows + g - 1) / g;     // positions of the rows
    const long long seen = ((long long)p.window + (span < p.K ? span : p.K) + TK - 2) / TK + 1 + ((long long)p.sinks + TK - 1) / TK;
    const long long behind = p.causal ? 0 : ((long long)p.K + TK - 1) / TK;
    if (seen + behind < tiles) tiles = seen + behind;
  }
  return tiles < 1 ? 1 : tiles;
}

SharePlan plan_shares(const sdllm_paged_attn_params& p, bool with_block, int tile_rows, int row_tiles, int TK, int at_once, int min_tiles) {
  const long long units = (long long)p.B * p.Hkv * row_tiles, tiles = paged_most_tiles(p, with_block, tile_rows, TK);
  const long long per = p.kv_splits > 0 ? (tiles + p.kv_splits - 1) / p.kv_splits : min_tiles;
  // A worker per unit where a unit is one share anyway, where the units go round all workers several times, and where finding the
  // shares (a walk over the batch's lengths) or the merge's grid would get long; and where the tiles of the 64 entries that are added up
  // at a time (entries) might not fit 32 bits
  const long long entries = (long long)p.B * row_tiles;
  if (p.kv_splits == 1 || tiles <= per || units * tile_rows >= (1 << 23) || entries > 2048 || (p.kv_splits == 0 && units >= 2LL * at_once) ||
      (entries < 64 ? entries : 64) * tiles >= (1LL << 31))
    return SharePlan{(int)units, 0};
  const long long w = (units * tiles + per - 1) / per, most = p.kv_splits > 0 ? 1 << 18 : at_once;
  return SharePlan{(int)(w < most ? w : most), (int)per};
}

size_t share_bytes(const SharePlan& pl, int tile_rows, int D) {
  return pl.min_tiles == 0 ? 0 : (size_t)pl.workers * 2 * tile_rows * (D + 2) * sizeof(float);
}

void set_shares(PagedArgs& a, const SharePlan& pl, int tile_rows, int row_tiles, int D, void* workspace) {
  a.tile_rows = tile_rows; a.row_tiles = row_tiles; a.by_row_tiles = FastDiv(row_tiles);
  a.workers = pl.workers; a.min_tiles = pl.min_tiles;
  a.ws_o = pl.min_tiles ? (float*)workspace : nullptr;
  a.ws_ml = pl.min_tiles ? a.ws_o + (size_t)pl.workers * 2 * tile_rows * D : nullptr;
}

static bool few_rows(const sdllm_paged_attn_params& p) { return (long long)p.Hq / p.Hkv * p.K <= 32; }

size_t paged_attention_workspace_bytes(const sdllm_paged_attn_params& p, bool with_block) {
  if (p.dtype == SDLLM_FP32) return paged_f32_workspace_bytes(p, with_block);
  return few_rows(p) ? paged_stream_workspace_bytes(p, with_block) : paged_tile_workspace_bytes(p, with_block);
}

hipError_t launch_paged_attention(const sdllm_paged_attn_params& p, const void* q, const void* k_pages, const void* v_pages,
                                  const int32_t* table, const int32_t* lens, const void* k_block, const void* v_block,
                                  const int32_t* q_lens, void* out, void* workspace, hipStream_t stream) {
  PagedArgs a{};
  a.q = q; a.kp = k_pages; a.vp = v_pages; a.table = table; a.lens = lens; a.kb = k_block; a.vb = v_block; a.q_lens = q_lens; a.out = out;
  dense_or(p.q_stride, p.Hq, p.K, p.D, a.q_st);
  dense_or(p.out_stride, p.Hq, p.K, p.D, a.o_st);
  dense_or(p.k_block_stride, p.Hkv, p.K, p.D, a.kb_st);
  dense_or(p.v_block_stride, p.Hkv, p.K, p.D, a.vb_st);
  a.B = p.B; a.Hq = p.Hq; a.Hkv = p.Hkv; a.g = p.Hq / p.Hkv; a.K = p.K; a.R = a.g * p.K;
  a.shift = __builtin_ctz(p.page_size); a.page_bytes = (unsigned)((long long)p.Hkv * p.page_size * p.D * (p.dtype == SDLLM_FP32 ? 4 : 2));
  a.n_pages = p.n_pages; a.max_pages = p.max_pages; a.max_kv = p.max_kv_len; a.causal = p.causal;
  // positions lie between -2^30 and 2^30: as far as the differences of two of them stay within 32 bits
  a.window = p.window < (1 << 30) ? p.window : 1 << 30; a.sinks = p.sinks < (1 << 30) ? p.sinks : 1 << 30;
  a.by_g = FastDiv(a.g); a.by_Hkv = FastDiv(a.Hkv);
  const float scale = p.scale > 0.f ? p.scale : 1.0f / sqrtf((float)p.D);
  a.scale_log2 = scale * kLog2e; a.thr8 = 8.0f / a.scale_log2;
  if (p.dtype == SDLLM_FP32) return launch_paged_f32(p, a, workspace, stream);
  return few_rows(p) ? launch_paged_stream(p, a, workspace, stream) : launch_paged_tile(p, a, workspace, stream);
}

}  // namespace sdllm
