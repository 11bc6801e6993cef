// Entry point of the attention over the paged cache: argument checks, the choice of kernel and of the number of key
// splits, and the kernel that joins the splits.
#include <algorithm>
#include <cmath>

#include "paged_cache.cuh"

namespace pd {
namespace paged {
namespace {

// out[row] = sum_z w_z O_z / sum_z w_z,  w_z = 2^(lse_z - max lse): a warp per (token, head), lanes across head_dim.
// HBM / L2-bound on the partial outputs, 4 bytes per element and split.
template <int D>
__global__ void __launch_bounds__(128) paged_attention_join(const Params p) {
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch_dependents();
  const int64_t rows = (int64_t)p.part_tokens * p.heads_q;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int h = (int)(row % p.heads_q);
  int t = (int)(row / p.heads_q);  // the place of a token's partial results
  // padding tokens, tokens beyond max_q_len, and places that a sequence does not fill have none
  if (p.part_by_sequence) {
    const int b = t / p.max_q_len;
    const Sequence seq = load_sequence(p, b);
    t -= b * p.max_q_len;
    if (t >= seq.n) return;
    t += seq.q0;
  } else {
    const int b = find_sequence(p.cu_q, p.batch, t);
    if (b >= p.batch || (unsigned)(t - __ldg(p.cu_q + b)) >= (unsigned)p.max_q_len) return;
  }
  const int per = D / 32;
  float lse_max = -INFINITY;
  for (int z = lane; z < p.splits; z += 32) lse_max = fmaxf(lse_max, p.part_lse[z * rows + row]);
  lse_max = warp_max(lse_max);
  float acc[per], sum = 0.f;
#pragma unroll
  for (int j = 0; j < per; ++j) acc[j] = 0.f;
  for (int z = 0; z < p.splits; ++z) {
    const float lse = p.part_lse[z * rows + row];
    if (lse == -INFINITY) continue;
    const float w = ex2(lse - lse_max);
    sum += w;
    const float* o = p.part_o + (z * rows + row) * D + lane * per;
#pragma unroll
    for (int j = 0; j < per; ++j) acc[j] += w * o[j];
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  uint32_t* out = reinterpret_cast<uint32_t*>(p.out + (int64_t)t * p.ld_out + (int64_t)h * D + lane * per);
#pragma unroll
  for (int j = 0; j < per; j += 2) out[j / 2] = pack_bf16(acc[j] * inv, acc[j + 1] * inv);
}

struct Plan {
  int rows_per_tile;            // 16, 32, 64: row kernel; 128 (head_dim 64), 256: chunk kernel
  int splits, min_split_tiles;  // in key tiles of the kernel (64, 128); the latter of the chunk kernels alone
  bool whole_items;
};

// Depends on the desc alone (the workspace size follows from it).
Plan plan(const pd_paged_attention_desc& d) {
  constexpr int kSms = 148;  // (not asked of the device: the workspace follows from the desc alone)
  Plan pl{};
  const int64_t group = d.heads_q / d.heads_kv, rows = std::min(d.max_q_len, d.tokens) * group;
  pl.rows_per_tile = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : d.head_dim == 64 ? 128 : 256;
  const bool chunk = pl.rows_per_tile > 64;
  const int64_t row_tiles = (rows + pl.rows_per_tile - 1) / pl.rows_per_tile;
  const int64_t items = row_tiles * d.heads_kv * d.batch;  // CTAs without splitting
  int64_t keys = d.max_kv_len;
  if (d.window > 0) keys = std::min<int64_t>(keys, (int64_t)d.window + d.sinks + d.max_q_len);
  const int64_t tile = !chunk ? 64 : d.head_dim == 64 ? 64 : 128, tiles = (keys + tile - 1) / tile;
  if (!chunk) {
    // two CTAs per SM share all key tiles evenly; fewer when there are not enough tiles for that
    pl.whole_items = tiles <= 2;
    const int64_t all = std::max<int64_t>(tiles, 1) * d.heads_kv * d.batch;  // (not 0: an empty batch launches nothing)
    pl.splits = (int)std::min<int64_t>(2 * kSms, all);
    return pl;
  }
  // One or four CTAs per SM, and splits only to fill the SMs, none below min_split_tiles.
  pl.min_split_tiles = d.head_dim == 64 ? 8 : 4;
  int64_t want = items > 0 ? kSms * (d.head_dim == 64 ? 4 : 1) / items : 1;
  want = std::min<int64_t>(want, (tiles + pl.min_split_tiles - 1) / pl.min_split_tiles);
  pl.splits = (int)std::min<int64_t>(std::max<int64_t>(want, 1), 256);
  return pl;
}

// Tokens that can have partial results in the chunk kernel (a token tensor may be padded to any length), at most d.tokens.
int64_t partial_tokens(const pd_paged_attention_desc& d) {
  return std::min<int64_t>(d.tokens, (int64_t)d.batch * std::min(d.max_q_len, d.tokens));
}
// Rows of partial results in the workspace, and entries of the piece table behind them.
size_t partial_rows(const pd_paged_attention_desc& d, const Plan& pl) {
  if (pl.rows_per_tile > 64) return pl.splits > 1 ? (size_t)pl.splits * partial_tokens(d) * d.heads_q : 0;
  return (size_t)2 * pl.splits * pl.rows_per_tile;
}
size_t table_entries(const pd_paged_attention_desc& d, const Plan& pl) {
  return pl.rows_per_tile > 64 ? 0 : (size_t)d.batch * d.heads_kv;
}
size_t workspace_bytes(const pd_paged_attention_desc& d) {
  const Plan pl = plan(d);
  return partial_rows(d, pl) * ((size_t)d.head_dim + 1) * sizeof(float) + table_entries(d, pl) * sizeof(int2);
}

}  // namespace
}  // namespace paged
}  // namespace pd

extern "C" size_t pd_attention_paged_workspace_bytes(const pd_paged_attention_desc* desc) {
  if (!desc || !pd::paged::valid(*desc) || !pd::paged::supported(*desc)) return 0;
  if (desc->batch == 0 || desc->tokens == 0 || desc->max_q_len == 0) return 0;
  return pd::paged::workspace_bytes(*desc);
}

extern "C" pd_status pd_attention_paged_fwd(const pd_paged_attention_desc* desc, const void* q, const void* k_cache,
                                            const void* v_cache, const int32_t* block_table, const int32_t* cu_q,
                                            const int32_t* kv_len, void* out, void* workspace, size_t workspace_bytes,
                                            cudaStream_t stream) {
  using namespace pd;
  if (!desc) return PD_ERR_NULL_POINTER;
  const pd_paged_attention_desc& d = *desc;
  if (!paged::valid(d)) return PD_ERR_BAD_SHAPE;
  if (!paged::supported(d)) return PD_ERR_UNSUPPORTED;
  const int64_t row = (int64_t)d.heads_q * d.head_dim;
  if (d.ld_q < row || d.ld_out < row || d.page_stride <= 0 || d.slot_stride <= 0 || d.head_stride <= 0)
    return PD_ERR_BAD_SHAPE;
  if (d.batch == 0 || d.tokens == 0 || d.max_q_len == 0) return PD_OK;
  if (!q || !k_cache || !v_cache || !block_table || !cu_q || !kv_len || !out) return PD_ERR_NULL_POINTER;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) ||
      ((d.ld_q | d.ld_out | d.page_stride | d.slot_stride | d.head_stride) & 7) != 0 ||
      ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(cu_q) |
        reinterpret_cast<uintptr_t>(kv_len)) & 3u) != 0)
    return PD_ERR_ALIGNMENT;
  const size_t need = paged::workspace_bytes(d);
  if (need > 0) {
    if (!workspace) return PD_ERR_NULL_POINTER;
    if (workspace_bytes < need) return PD_ERR_WORKSPACE_TOO_SMALL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return PD_ERR_ALIGNMENT;
  }
  if (pd_status st = require_sm100(); st != PD_OK) return st;

  const paged::Plan pl = paged::plan(d);
  paged::Params p{};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.block_table = block_table; p.cu_q = cu_q; p.kv_len = kv_len;
  p.status = device_status_ptr();
  if (!p.status) return PD_ERR_CUDA;
  p.wait_limit_ns = debug_wait_limit_ns(); p.withhold_loads = debug_withhold_loads();
  p.ld_q = d.ld_q; p.ld_out = d.ld_out;
  p.batch = d.batch; p.tokens = d.tokens; p.heads_q = d.heads_q; p.heads_kv = d.heads_kv; p.group = d.heads_q / d.heads_kv;
  p.num_pages = d.num_pages; p.page_size = d.page_size; p.max_pages = d.max_pages;
  while ((1 << p.page_shift) < d.page_size) ++p.page_shift;
  p.max_q_len = std::min(d.max_q_len, d.tokens); p.window = std::min(d.window, paged::kMaxPositions); p.sinks = d.sinks;
  p.part_tokens = (int)paged::partial_tokens(d); p.part_by_sequence = p.part_tokens < d.tokens;
  p.splits = pl.splits; p.min_split_tiles = pl.min_split_tiles; p.whole_items = pl.whole_items;
  p.scale_log2e = paged::base2_scale(d.scale);
  if (need > 0) {
    const size_t rows = paged::partial_rows(d, pl);  // (an even number in the row kernel: the table is aligned)
    p.part_o = static_cast<float*>(workspace);
    p.part_lse = p.part_o + rows * d.head_dim;
    p.pieces = reinterpret_cast<int2*>(p.part_lse + rows);
  }
  logf("paged attention batch %d tokens %d (max %d) heads %d/%d x %d: tiles of %d rows, %s %d", d.batch, d.tokens,
       d.max_q_len, d.heads_q, d.heads_kv, d.head_dim, pl.rows_per_tile, pl.rows_per_tile > 64 ? "key splits" : "CTAs", pl.splits);
  const pd_status launched = pl.rows_per_tile > 64 ? paged::launch_chunk(d, p, k_cache, v_cache, stream)
                                                     : paged::launch_rows(d, p, k_cache, v_cache, pl.rows_per_tile, stream);
  if (launched != PD_OK) return launched;
  if (pl.rows_per_tile > 64 && pl.splits > 1) {
    const int64_t rows = (int64_t)p.part_tokens * d.heads_q;
    const unsigned grid = (unsigned)((rows + 3) / 4);
    if (d.head_dim == 64) launch_pdl(paged::paged_attention_join<64>, dim3(grid), dim3(128), 0, stream, p);
    else launch_pdl(paged::paged_attention_join<128>, dim3(grid), dim3(128), 0, stream, p);
    return check_launch();
  }
  return PD_OK;
}
