// Attention over an 8-bit paged cache: a warp per token and query head walks the keys that the token sees.
#include "cache_q8.cuh"

namespace pd {
namespace paged {
namespace {

template <pd_dtype T, int D>
__global__ void __launch_bounds__(128) paged_attention_q8_kernel(const Params p, const uint8_t* k_cache, const uint8_t* v_cache,
                                                                 int64_t page_stride, int64_t slot_stride, int64_t head_stride,
                                                                 const Scales scales) {
  griddep_wait();
  griddep_launch_dependents();
  constexpr int kPer = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= (int64_t)p.tokens * p.heads_q) return;
  const int t = (int)(row / p.heads_q), h = (int)(row % p.heads_q), kvh = h / p.group;
  const int b = find_sequence(p.cu_q, p.batch, t);
  if (b >= p.batch) return;
  const Sequence seq = load_sequence(p, b);
  if (t < seq.q0 || t - seq.q0 >= seq.n) return;
  const int pos = seq.pos0 + (t - seq.q0);
  float q[kPer], o[kPer], m = -INFINITY, l = 0.f;
  for (int j = 0; j < kPer; ++j) {
    q[j] = __bfloat162float(p.q[(int64_t)t * p.ld_q + (int64_t)h * D + lane * kPer + j]);
    o[j] = 0.f;
  }
  const int end = min(pos + 1, seq.length);
  for (int key = 0; key < end; ++key) {
    if (p.window > 0 && key <= pos - p.window && key >= p.sinks) continue;
    const int page = page_of(p, b, key), slot = key & (p.page_size - 1);
    float k[kPer], v[kPer], ks = 0.f, vs = 0.f;
    for (int j = 0; j < kPer; ++j) k[j] = v[j] = 0.f;
    if (page < p.num_pages) {
      const int64_t at = page * page_stride + slot * slot_stride + kvh * head_stride + lane * kPer;
      for (int j = 0; j < kPer; j += 2) {
        const float2 a = q8_pair_to_float<T>(*reinterpret_cast<const uint16_t*>(k_cache + at + j));
        const float2 c = q8_pair_to_float<T>(*reinterpret_cast<const uint16_t*>(v_cache + at + j));
        k[j] = a.x; k[j + 1] = a.y; v[j] = c.x; v[j + 1] = c.y;
      }
      ks = scales.k[scales.at(page, kvh, slot)];
      vs = scales.v[scales.at(page, kvh, slot)];
    }
    float s = 0.f;
    for (int j = 0; j < kPer; ++j) s = fmaf(q[j], k[j], s);
    s = warp_sum(s) * ks * p.scale_log2e;
    const float top = fmaxf(m, s), alpha = exp2f(m - top), e = exp2f(s - top);
    m = top;
    l = l * alpha + e;
    for (int j = 0; j < kPer; ++j) o[j] = fmaf(e * vs, v[j], o[j] * alpha);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  for (int j = 0; j < kPer; ++j) p.out[(int64_t)t * p.ld_out + (int64_t)h * D + lane * kPer + j] = __float2bfloat16_rn(o[j] * inv);
}

inline Plan plan_q8(const pd_paged_attention_desc& d) { return plan(d, 8); }

}  // namespace
}  // namespace paged
}  // namespace pd

extern "C" size_t pd_attention_paged_q8_workspace_bytes(const pd_paged_attention_desc* desc) {
  if (!desc || !pd::paged::valid(*desc) || !pd::paged::supported(*desc)) return 0;
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
  if (!paged::supported(d)) return PD_ERR_UNSUPPORTED;
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
  if (pl.rows_per_tile <= 64) return paged::launch_rows_q8(d, p, scales->dtype, sc, k_cache, v_cache, pl.rows_per_tile, stream);
  const bool i8 = scales->dtype == PD_I8;
  auto kernel = d.head_dim == 64 ? (i8 ? paged::paged_attention_q8_kernel<PD_I8, 64> : paged::paged_attention_q8_kernel<PD_E4M3, 64>)
                                 : (i8 ? paged::paged_attention_q8_kernel<PD_I8, 128> : paged::paged_attention_q8_kernel<PD_E4M3, 128>);
  launch_pdl(kernel, dim3((unsigned)(((int64_t)d.tokens * d.heads_q + 3) / 4)), dim3(128), 0, stream, p, static_cast<const uint8_t*>(k_cache),
             static_cast<const uint8_t*>(v_cache), d.page_stride, d.slot_stride, d.head_stride, sc);
  return check_launch();
}
