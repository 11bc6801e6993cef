// Entry point of the attention over an 8-bit paged cache: argument checks and the choice of kernel.
#include "cache_q8.cuh"
#include "paged_join.cuh"

namespace pd {
namespace paged {
namespace {

// (the row kernel's tiles can be of 32 keys, and all of a batch's are counted in 32 bits)
bool supported_q8(const pd_paged_attention_desc& d) {
  return supported(d) && (int64_t)d.batch * d.heads_kv * (((int64_t)d.max_pages * d.page_size + 31) / 32) <= kMaxPositions;
}

// Row kernel: up to four warps beside each other take cache heads (the rows of a slot that lie beside each other in the usual
// layout), as many as divide the heads; the rest of the four share keys, or rows.
//   17 to 24 rows: tiles of 24 have a quarter less to compute than tiles of 32, but twice the heads to an item, so twice the
//   partial results at the ends of a CTA's share.  So 24 where shares are long, counted in tiles of 128 keys and heads (20 rows, 8 heads,
//   tiles of 24 against 32):
//     head_dim 64, from 12 on:  64 x 4096 keys (55) 107 against 133 us, 64 x 1024 (14) 45 and 49, 8 x 8192 (14) 42 and 45; but 16 x 2048 (7)
//       30 and 29, 8 x 1024 (2) 18 and 16
//     head_dim 128, from 32 on: 64 x 4096 (55) 199 against 222, 32 x 4096 (28) 115 and 121; but 32 x 2048 (14) 76 and 72, 16 x 2048 (7) 53 and 43.
//       Lengths are usually well below max_kv_len, which alone is known here: hence 32, although 28 full tiles would do.
//   65 rows and more: the chunk kernel (64 x 4096 keys, 8 heads of 128: 450 us for 68 rows, 476 for 256, where tiles of 64 rows take 428
//   for 64, of 32 rows 231 for 32).
Plan plan_q8(const pd_paged_attention_desc& d) {
  Plan pl{};
  const int64_t rows = plan_rows(d);
  const bool long_shares = plan_keys(d) * d.heads_kv * d.batch >= (int64_t)(d.head_dim == 64 ? 12 : 32) * 128 * 2 * kSms;
  const bool rows24 = rows > 16 && rows <= 24 && long_shares;
  pl.rows_per_tile = rows <= 8 ? 8 : rows <= 16 ? 16 : rows24 ? 24 : rows <= 32 ? 32 : rows <= 64 ? 64 : 256;
  if (pl.rows_per_tile > 64) {
    plan_splits(d, pl);
    return pl;
  }
  const int warps = pl.rows_per_tile <= 24 ? 4 : pl.rows_per_tile == 32 ? 2 : 1;  // that have different heads or keys
  pl.heads_per_item = warps;
  while (d.heads_kv % pl.heads_per_item != 0) pl.heads_per_item /= 2;
  pl.tile = 32 * warps / pl.heads_per_item;
  plan_shares(d, pl);
  return pl;
}

}  // namespace
}  // namespace paged
}  // namespace pd

extern "C" size_t pd_attention_paged_q8_workspace_bytes(const pd_paged_attention_desc* desc) {
  if (!desc || !pd::paged::valid(*desc) || !pd::paged::supported_q8(*desc)) return 0;
  if (desc->batch == 0 || desc->tokens == 0 || desc->max_q_len == 0) return 0;
  return pd::paged::workspace_bytes(*desc, pd::paged::plan_q8(*desc));
}

extern "C" pd_status pd_attention_paged_q8_fwd(const pd_paged_attention_desc* desc, const pd_cache_scales* scales, const void* q,
                                               const void* k_cache, const void* v_cache, const int32_t* block_table,
                                               const int32_t* cu_q, const int32_t* kv_len, void* out, void* workspace,
                                               size_t workspace_bytes, cudaStream_t stream) {
  using namespace pd;
  if (!desc || !scales) return PD_ERR_NULL_POINTER;
  const pd_paged_attention_desc& d = *desc;
  if (!paged::valid(d) || !paged::q8_dtype(scales->dtype) || !paged::q8_block_valid(scales->block, d.page_size)) return PD_ERR_BAD_SHAPE;
  if (!paged::supported_q8(d)) return PD_ERR_UNSUPPORTED;
  const int64_t row = (int64_t)d.heads_q * d.head_dim;
  if (d.ld_q < row || d.ld_out < row || d.page_stride <= 0 || d.slot_stride <= 0 || d.head_stride <= 0) return PD_ERR_BAD_SHAPE;
  if (d.batch == 0 || d.tokens == 0 || d.max_q_len == 0) return PD_OK;
  if (!q || !k_cache || !v_cache || !scales->k_scale || !scales->v_scale || !block_table || !cu_q || !kv_len || !out) return PD_ERR_NULL_POINTER;
  auto bits = [](const void* v) { return reinterpret_cast<uintptr_t>(v); };
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || ((d.ld_q | d.ld_out) & 7) != 0 ||
      ((d.page_stride | d.slot_stride | d.head_stride) & 15) != 0 ||
      ((bits(block_table) | bits(cu_q) | bits(kv_len) | bits(scales->k_scale) | bits(scales->v_scale)) & 3u) != 0)
    return PD_ERR_ALIGNMENT;
  const paged::Plan pl = paged::plan_q8(d);
  const size_t need = paged::workspace_bytes(d, pl);
  if (need > 0) {
    if (!workspace) return PD_ERR_NULL_POINTER;
    if (workspace_bytes < need) return PD_ERR_WORKSPACE_TOO_SMALL;
    if ((bits(workspace) & 255u) != 0) return PD_ERR_ALIGNMENT;
  }
  if (pd_status st = require_sm100(); st != PD_OK) return st;
  paged::Params p = paged::make_params(d, pl, q, block_table, cu_q, kv_len, out, workspace);
  if (!p.status) return PD_ERR_CUDA;
  const paged::Scales sc = paged::make_scales(*scales, d.heads_kv, d.page_size);
  logf("paged attention (%s) batch %d tokens %d (max %d) heads %d/%d x %d: tiles of %d rows, %s %d", scales->dtype == PD_I8 ? "int8" : "e4m3",
       d.batch, d.tokens, d.max_q_len, d.heads_q, d.heads_kv, d.head_dim, pl.rows_per_tile, pl.rows_per_tile > 64 ? "key splits" : "CTAs", pl.splits);
  if (pl.rows_per_tile <= 64)
    return scales->dtype == PD_I8 ? paged::launch_rows_i8(d, p, pl, sc, k_cache, v_cache, stream) : paged::launch_rows_e4m3(d, p, pl, sc, k_cache, v_cache, stream);
  if (pd_status st = paged::launch_chunk_q8(d, p, scales->dtype, sc, k_cache, v_cache, stream); st != PD_OK) return st;
  return pl.splits > 1 ? paged::launch_join(d, p, stream) : PD_OK;
}
