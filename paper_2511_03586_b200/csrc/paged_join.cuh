// The kernel that joins the key splits of the chunk kernels of the paged attention, and its launch.  Internal to the library.
#pragma once

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

inline pd_status launch_join(const pd_paged_attention_desc& d, const Params& p, cudaStream_t stream) {
  const int64_t rows = (int64_t)p.part_tokens * d.heads_q;
  const unsigned grid = (unsigned)((rows + 3) / 4);
  if (d.head_dim == 64) launch_pdl(paged_attention_join<64>, dim3(grid), dim3(128), 0, stream, p);
  else launch_pdl(paged_attention_join<128>, dim3(grid), dim3(128), 0, stream, p);
  return check_launch();
}

}  // namespace
}  // namespace paged
}  // namespace pd
