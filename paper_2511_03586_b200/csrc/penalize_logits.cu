// Penalties for repeated tokens, biases and grammar masks on rows of logits, in one pass over them:
//
//   z = logits[i, j]
//   z = z > 0 ? z / r_i : z * r_i                        where j occurs in row i's history
//   z = z - f_i * n_ij - g_i * [n_ij > 0]                n_ij: how often j occurs behind the prompt
//   z = z + bias_ij                                      the last entry of row i's list that names j
//   z = -inf                                             where row i's mask has bit j cleared
//
// Bound: HBM, every logit read once and written once.  A CTA takes 16 logits a thread of one row and has them copied to shared
// memory (every thread its own, asynchronously); while they are under way it counts the row's history in shared memory, one word for each of its tokens:
//   bit 31: occurs in the history;  bits 11 ... 30: times behind the prompt;  bits 0 ... 10: 1 + entry of the bias list
// The counts are integer sums, the entries a maximum, so neither depends on the order in which threads get there.  Every CTA of
// a row reads the whole history (from the L2 cache, 16 times 32 KB for 8000 tokens of a row of 128000 logits), 16 tokens a thread at
// a time; a row that changes nothing skips the counting.
//   256 x 128000 fp32 with up to 8000 tokens a row: 91 us with the logits in registers and four tokens at a time, 150 with the
//   history shared out over a cluster (half of a text's tokens belong to few slices, and additions to another CTA's shared memory
//   queue there).
#include "pd_common.cuh"

namespace pd {
namespace {

constexpr int kEach = 16;  // logits per thread
constexpr uint32_t kOccurs = 0x80000000u, kOnce = 1u << 11, kBiasBits = kOnce - 1;

struct PenaltyParams {
  const void* logits;
  void* out;
  const int32_t *history, *history_len, *prompt_len;
  const float *repetition, *frequency, *presence;
  const int32_t* bias_tokens;
  const float* bias_values;
  const uint32_t* mask;
  const int32_t* mask_row;
  int64_t ld, ld_out, ld_history, ld_mask;
  int vocab, history_cols, bias_cols, mask_rows;
  int slices;  // CTAs of a row
  int vectors; // rows of logits and of results begin on 16-byte boundaries
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* to, float v) { *to = v; }
__device__ __forceinline__ void put(__nv_bfloat16* to, float v) { *to = __float2bfloat16_rn(v); }

template <typename In, typename Out, int THREADS>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) penalize_logits_kernel(const PenaltyParams p) {
  constexpr int kSlice = THREADS * kEach;
  constexpr int kQuad = 4 * sizeof(In);
  extern __shared__ __align__(16) uint32_t words[];
  In* logits = reinterpret_cast<In*>(words + kSlice);
  griddep_wait();
  griddep_launch_dependents();
  const int row = blockIdx.x / p.slices, first = (blockIdx.x % p.slices) * kSlice;
  const int n = min(kSlice, p.vocab - first);
  const In* src = static_cast<const In*>(p.logits) + (int64_t)row * p.ld + first;
  Out* dst = static_cast<Out*>(p.out) + (int64_t)row * p.ld_out + first;

  // this thread's logits: four at a time, THREADS * 4 apart
#pragma unroll
  for (int k = 0; k < kEach / 4; ++k) {
    const int j = (k * THREADS + threadIdx.x) * 4;
    if (p.vectors && j + 4 <= n)
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(logits + j)), "l"(src + j), "n"(kQuad) : "memory");
  }
  float r = p.repetition ? p.repetition[row] : 1.f;
  if (!(r > 0.f && r <= 3.402823466e38f && 1.f / r <= 3.402823466e38f)) r = 1.f;
  const float inv = 1.f / r;
  const float f = p.frequency ? p.frequency[row] : 0.f, g = p.presence ? p.presence[row] : 0.f;
  const int length = p.history ? min(max(p.history_len ? p.history_len[row] : p.history_cols, 0), p.history_cols) : 0;
  const int prompt = p.prompt_len ? p.prompt_len[row] : 0;
  const int mask_row = !p.mask ? -1 : p.mask_row ? p.mask_row[row] : row;
  const bool masked = mask_row >= 0 && mask_row < p.mask_rows;
  const bool counts = length > 0 && (r != 1.f || f != 0.f || g != 0.f);
  const bool changes = counts || p.bias_cols > 0;  // (the same for all threads)
  if (changes) {
#pragma unroll
    for (int k = 0; k < kEach / 4; ++k) *reinterpret_cast<uint4*>(words + (k * THREADS + threadIdx.x) * 4) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (p.bias_cols > 0) {
      for (int e = threadIdx.x; e < p.bias_cols; e += THREADS) {
        const uint32_t at = (uint32_t)p.bias_tokens[(int64_t)row * p.bias_cols + e] - (uint32_t)first;
        if (at < (uint32_t)n) atomicMax(words + at, (uint32_t)e + 1u);
      }
      __syncthreads();
    }
    if (counts) {
      const int32_t* history = p.history + (int64_t)row * p.ld_history;
      constexpr int kAhead = 16;
      for (int h0 = threadIdx.x; h0 < length; h0 += kAhead * THREADS) {
        int32_t token[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) token[k] = h0 + k * THREADS < length ? history[h0 + k * THREADS] : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const uint32_t at = (uint32_t)token[k] - (uint32_t)first;
          if (at < (uint32_t)n) {
            if (h0 + k * THREADS >= prompt) atomicAdd(words + at, kOnce);
            else atomicOr(words + at, kOccurs);
          }
        }
      }
      __syncthreads();
    }
  }
  const uint32_t* mask = p.mask + (int64_t)mask_row * p.ld_mask;
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int k = 0; k < kEach / 4; ++k) {
    const int j = (k * THREADS + threadIdx.x) * 4;
    if (j >= n) break;
    const bool quad = p.vectors && j + 4 <= n;
    float z[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = quad ? as_float(logits[j + e]) : j + e < n ? as_float(src[j + e]) : 0.f;
    if (changes) {
      const uint4 w4 = *reinterpret_cast<const uint4*>(words + j);
      if (w4.x | w4.y | w4.z | w4.w) {
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        // (few instructions and one branch: in a row with a history most warps come through here.  With a division, and a branch for
        // every case, this took 30 of 89 us.)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t times = (w[e] & ~kOccurs) / kOnce;
          z[e] *= w[e] < kOnce ? 1.f : z[e] > 0.f ? inv : r;
          z[e] = times > 0 ? fmaf(-f, (float)times, z[e]) - g : z[e];
        }
        if ((w[0] | w[1] | w[2] | w[3]) & kBiasBits) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (w[e] & kBiasBits) z[e] += p.bias_values[(int64_t)row * p.bias_cols + (w[e] & kBiasBits) - 1];
        }
      }
    }
    if (masked) {
      const uint32_t allowed = __ldg(mask + (first + j) / 32) >> (j % 32);  // (the four lie in one word)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!((allowed >> e) & 1u)) z[e] = -INFINITY;
    }
    if (quad) {
      store_out4(dst, j / 4, make_float4(z[0], z[1], z[2], z[3]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < n) put(dst + j + e, z[e]);
    }
  }
}

template <typename In, typename Out>
pd_status launch(PenaltyParams& p, int64_t rows, cudaStream_t s) {
  // 512 threads, 8192 logits per CTA; 128 and 2048 where that would leave SMs without work
  const bool narrow = rows * ((p.vocab + 8191) / 8192) < 2 * 148;
  const int slice = narrow ? 2048 : 8192;
  p.slices = (p.vocab + slice - 1) / slice;
  if (rows * p.slices > 0x7fffffff) return PD_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(rows * p.slices));
  const size_t smem = (size_t)slice * (4 + sizeof(In));
  if (narrow) {
    launch_pdl(penalize_logits_kernel<In, Out, 128>, grid, dim3(128), smem, s, p);
  } else {
    static PerDeviceFlag smem_allowed;
    if (pd_status st = allow_dynamic_smem(penalize_logits_kernel<In, Out, 512>, (int)smem, smem_allowed); st != PD_OK) return st;
    launch_pdl(penalize_logits_kernel<In, Out, 512>, grid, dim3(512), smem, s, p);
  }
  return check_launch();
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_penalize_logits(const pd_penalize_desc* desc, const void* logits, void* out, const int32_t* history,
                                        const int32_t* history_len, const int32_t* prompt_len, const float* repetition,
                                        const float* frequency, const float* presence, const int32_t* bias_tokens,
                                        const float* bias_values, const uint32_t* mask, const int32_t* mask_row,
                                        cudaStream_t stream) {
  if (!desc) return PD_ERR_NULL_POINTER;
  const pd_penalize_desc& d = *desc;
  auto is_dtype = [](pd_dtype t) { return t == PD_BF16 || t == PD_F32; };
  if (d.rows < 0 || d.vocab <= 0 || !is_dtype(d.dtype) || !is_dtype(d.out_dtype) || d.ld_logits < d.vocab || d.ld_out < d.vocab ||
      d.history_cols < 0 || d.bias_cols < 0 || d.mask_rows < 0)
    return PD_ERR_BAD_SHAPE;
  const int64_t words = (d.vocab + 31) / 32;
  if ((history && d.ld_history < d.history_cols) || (mask && d.ld_mask < words)) return PD_ERR_BAD_SHAPE;
  if (d.vocab > (1 << 24) || d.rows > 0x7fffffff || d.history_cols >= (1 << 20) || d.bias_cols > (int64_t)pd::kBiasBits) return PD_ERR_UNSUPPORTED;
  if (d.rows == 0) return PD_OK;
  if (!logits || !out || (d.bias_cols > 0 && (!bias_tokens || !bias_values))) return PD_ERR_NULL_POINTER;
  if (mask && !mask_row && d.mask_rows < d.rows) return PD_ERR_BAD_SHAPE;
  auto bits = [](const void* v) { return reinterpret_cast<uintptr_t>(v); };
  const int64_t in_size = d.dtype == PD_F32 ? 4 : 2, out_size = d.out_dtype == PD_F32 ? 4 : 2;
  if ((bits(logits) & (uintptr_t)(in_size - 1)) || (bits(out) & (uintptr_t)(out_size - 1)) ||
      ((bits(history) | bits(history_len) | bits(prompt_len) | bits(repetition) | bits(frequency) | bits(presence) | bits(bias_tokens) |
        bits(bias_values) | bits(mask) | bits(mask_row)) & 3u) != 0)
    return PD_ERR_ALIGNMENT;
  if (pd_status st = pd::require_sm100(); st != PD_OK) return st;
  pd::PenaltyParams p{};
  p.logits = logits; p.out = out;
  p.history = d.history_cols > 0 ? history : nullptr; p.history_len = history_len; p.prompt_len = prompt_len;
  p.repetition = repetition; p.frequency = frequency; p.presence = presence;
  p.bias_tokens = bias_tokens; p.bias_values = bias_values; p.mask = mask; p.mask_row = mask_row;
  p.ld = d.ld_logits; p.ld_out = d.ld_out; p.ld_history = d.ld_history; p.ld_mask = d.ld_mask;
  p.vocab = (int)d.vocab; p.history_cols = (int)d.history_cols; p.bias_cols = (int)d.bias_cols;
  p.mask_rows = (int)(d.mask_rows < 0x7fffffff ? d.mask_rows : 0x7fffffff);
  p.vectors = ((bits(logits) | (uintptr_t)(d.ld_logits * in_size)) & (uintptr_t)(4 * in_size - 1)) == 0 &&
              ((bits(out) | (uintptr_t)(d.ld_out * out_size)) & (uintptr_t)(4 * out_size - 1)) == 0;
  pd::logf("penalize logits: %lld x %lld, history of %lld, %lld biases", (long long)d.rows, (long long)d.vocab, (long long)d.history_cols, (long long)d.bias_cols);
  if (d.dtype == PD_F32)
    return d.out_dtype == PD_F32 ? pd::launch<float, float>(p, d.rows, stream) : pd::launch<float, __nv_bfloat16>(p, d.rows, stream);
  return d.out_dtype == PD_F32 ? pd::launch<__nv_bfloat16, float>(p, d.rows, stream) : pd::launch<__nv_bfloat16, __nv_bfloat16>(p, d.rows, stream);
}
