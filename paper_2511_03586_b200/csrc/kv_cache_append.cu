// Appends the new tokens' keys and values to the paged cache:
//
//   cache[block_table[b, p / page_size], p % page_size, :, :] = new[t, :, :]
//
// for token t of sequence b at position p = kv_len[b] - n_b + (t - cu_q[b]).  A copy: HBM-bound for prompts (2 x 2
// bytes per element of K and V each way), one launch and one chain of dependent loads (cu_q, kv_len, block_table)
// for a decode batch.
//
// One warp looks its token's sequence up (a 32-way search of cu_q by all lanes, so that a batch of up to 32 takes one
// step) and copies its share of the token's K and V with 16-byte accesses.
#include "paged_cache.cuh"

namespace pd {
namespace {

struct AppendParams {
  const uint4 *k_new, *v_new;
  uint4 *k_cache, *v_cache;
  const int32_t *block_table, *cu_q, *kv_len;
  int64_t ld_new, page_stride, slot_stride, head_stride;  // in units of 16 bytes
  int batch, tokens, heads, head_vecs;                    // head_vecs: 16-byte units of a head
  int num_pages, page_size, max_pages;
};

constexpr int kWarps = 4;
constexpr int kMaxIndex = 1 << 30;  // of tokens and sequences: sums with a search's steps stay in 32 bits

__global__ void __launch_bounds__(32 * kWarps) kv_cache_append_kernel(const AppendParams p) {
  const int lane = threadIdx.x & 31;
  const int t = blockIdx.x * kWarps + (threadIdx.x >> 5);
  griddep_wait();
  griddep_launch_dependents();
  if (t >= p.tokens) return;
  // the token's data does not depend on where it goes: fetch the first part before the lookups
  const int vecs = p.heads * p.head_vecs;  // per tensor
  const uint4* ks = p.k_new + (int64_t)t * p.ld_new;
  const uint4* vs = p.v_new + (int64_t)t * p.ld_new;
  constexpr int kAhead = 4;  // 32 lanes x 4 x 16 bytes: 1024 elements of K and of V
  uint4 kd[kAhead], vd[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int c = lane + 32 * i;
    if (c < vecs) { kd[i] = __ldcs(ks + c); vd[i] = __ldcs(vs + c); }
  }
  const int b = paged::find_sequence(p.cu_q, p.batch, t);
  if (b >= p.batch || t < __ldg(p.cu_q + b)) return;  // padding behind the last sequence
  const int pos = max(__ldg(p.kv_len + b), 0) - (__ldg(p.cu_q + b + 1) - t);
  if (pos < 0) return;
  const int index = pos / p.page_size, slot = pos - index * p.page_size;
  if (index >= p.max_pages) return;
  const int page = __ldg(p.block_table + (int64_t)b * p.max_pages + index);
  if ((unsigned)page >= (unsigned)p.num_pages) return;
  const int64_t base = (int64_t)page * p.page_stride + (int64_t)slot * p.slot_stride;
  auto offset = [&](int c) {
    const int head = c / p.head_vecs;
    return base + (int64_t)head * p.head_stride + (c - head * p.head_vecs);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int c = lane + 32 * i;
    if (c < vecs) {
      const int64_t o = offset(c);
      p.k_cache[o] = kd[i];
      p.v_cache[o] = vd[i];
    }
  }
  for (int c = lane + 32 * kAhead; c < vecs; c += 32) {
    const int64_t o = offset(c);
    const uint4 a = __ldcs(ks + c), b4 = __ldcs(vs + c);
    p.k_cache[o] = a;
    p.v_cache[o] = b4;
  }
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_kv_cache_append(const pd_paged_attention_desc* desc, const void* k_new, const void* v_new,
                                        int64_t ld_new, void* k_cache, void* v_cache, const int32_t* block_table,
                                        const int32_t* cu_q, const int32_t* kv_len, cudaStream_t stream) {
  if (!desc) return PD_ERR_NULL_POINTER;
  const pd_paged_attention_desc& d = *desc;
  if (d.batch < 0 || d.tokens < 0) return PD_ERR_BAD_SHAPE;
  if (d.heads_kv <= 0 || d.head_dim <= 0 || d.num_pages <= 0 || d.page_size <= 0 || d.max_pages <= 0) return PD_ERR_BAD_SHAPE;
  if (d.head_dim % 8 != 0 || d.head_dim > 1024 || d.heads_kv > 65536 || d.batch > pd::kMaxIndex || d.tokens > pd::kMaxIndex)
    return PD_ERR_UNSUPPORTED;
  if (ld_new < (int64_t)d.heads_kv * d.head_dim) return PD_ERR_BAD_SHAPE;
  if (d.page_stride <= 0 || d.slot_stride <= 0 || d.head_stride <= 0) return PD_ERR_BAD_SHAPE;
  if (d.batch == 0 || d.tokens == 0) return PD_OK;
  if (!k_new || !v_new || !k_cache || !v_cache || !block_table || !cu_q || !kv_len) return PD_ERR_NULL_POINTER;
  if (!pd::aligned16(k_new) || !pd::aligned16(v_new) || !pd::aligned16(k_cache) || !pd::aligned16(v_cache) ||
      ((ld_new | d.page_stride | d.slot_stride | d.head_stride) & 7) != 0 ||
      ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(cu_q) |
        reinterpret_cast<uintptr_t>(kv_len)) & 3u) != 0)
    return PD_ERR_ALIGNMENT;
  if (pd_status st = pd::require_sm100(); st != PD_OK) return st;
  pd::AppendParams p{};
  p.k_new = static_cast<const uint4*>(k_new);
  p.v_new = static_cast<const uint4*>(v_new);
  p.k_cache = static_cast<uint4*>(k_cache);
  p.v_cache = static_cast<uint4*>(v_cache);
  p.block_table = block_table; p.cu_q = cu_q; p.kv_len = kv_len;
  p.ld_new = ld_new / 8; p.page_stride = d.page_stride / 8; p.slot_stride = d.slot_stride / 8;
  p.head_stride = d.head_stride / 8;
  p.batch = d.batch; p.tokens = d.tokens; p.heads = d.heads_kv; p.head_vecs = d.head_dim / 8;
  p.num_pages = d.num_pages; p.page_size = d.page_size; p.max_pages = d.max_pages;
  pd::logf("kv cache append: %d tokens of %d sequences", d.tokens, d.batch);
  pd::launch_pdl(pd::kv_cache_append_kernel, dim3((d.tokens + pd::kWarps - 1) / pd::kWarps), dim3(32 * pd::kWarps), 0,
                 stream, p);
  return pd::check_launch();
}
