// Entry point of the attention over the paged cache: argument checks, the choice of kernel and of the number of key
// splits.
#include "paged_join.cuh"

extern "C" size_t pd_attention_paged_workspace_bytes(const pd_paged_attention_desc* desc) {
  if (!desc || !pd::paged::valid(*desc) || !pd::paged::supported(*desc)) return 0;
  if (desc->batch == 0 || desc->tokens == 0 || desc->max_q_len == 0) return 0;
  return pd::paged::workspace_bytes(*desc, pd::paged::plan(*desc));
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
  const paged::Plan pl = paged::plan(d);
  const size_t need = paged::workspace_bytes(d, pl);
  if (need > 0) {
    if (!workspace) return PD_ERR_NULL_POINTER;
    if (workspace_bytes < need) return PD_ERR_WORKSPACE_TOO_SMALL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return PD_ERR_ALIGNMENT;
  }
  if (pd_status st = require_sm100(); st != PD_OK) return st;

  paged::Params p = paged::make_params(d, pl, q, block_table, cu_q, kv_len, out, workspace);
  if (!p.status) return PD_ERR_CUDA;
  logf("paged attention batch %d tokens %d (max %d) heads %d/%d x %d: tiles of %d rows, %s %d", d.batch, d.tokens,
       d.max_q_len, d.heads_q, d.heads_kv, d.head_dim, pl.rows_per_tile, pl.rows_per_tile > 64 ? "key splits" : "CTAs", pl.splits);
  const pd_status launched = pl.rows_per_tile > 64 ? paged::launch_chunk(d, p, k_cache, v_cache, stream)
                                                     : paged::launch_rows(d, p, k_cache, v_cache, pl.rows_per_tile, stream);
  if (launched != PD_OK) return launched;
  if (pl.rows_per_tile > 64 && pl.splits > 1) return paged::launch_join(d, p, stream);
  return PD_OK;
}
