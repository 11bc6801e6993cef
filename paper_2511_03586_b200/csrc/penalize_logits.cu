// Penalties for repeated tokens, biases and grammar masks on rows of logits, in one pass over them:
//
//   z = logits[i, j]
//   z = z > 0 ? z / r_i : z * r_i                        where j occurs in row i's history
//   z = z - f_i * n_ij - g_i * [n_ij > 0]                n_ij: how often j occurs behind the prompt
//   z = z + bias_ij                                      the last entry of row i's list that names j
//   z = -inf                                             where row i's mask has bit j cleared
//
// Bound: HBM, every logit read once and written once.  A CTA takes a slice of one row, 32 logits a thread (16 where there are few rows), which
// it loads first; while they are under way it counts the row's history, in a word of shared memory for each of the slice's tokens:
//   bit 31: occurs in the history;  bits 11 ... 30: times behind the prompt;  bits 0 ... 10: 1 + entry of the bias list
// The counts are integer sums, the entries a maximum, so neither depends on the order in which threads get there.  Every CTA of a
// row reads the whole history, from the L2 cache.  A row that changes nothing skips the counting.
//   256 x 128000 fp32, up to 8000 tokens a row, half of the rows masked: 68 us in long runs (3.9 TB/s), 45 to 49 without histories and biases.
//   A single call takes 75.  Other forms, single, when this one took 76: slices half as long (twice as many looks at the history) 82; several slices to a CTA, their logits copied ahead, 80; a plain copy first
//   and the named tokens mended one by one after it 100; the history shared out over a cluster 150 (half of a text's tokens
//   belong to few slices, and additions to another CTA's shared memory queue there).
#include "pd_common.cuh"

namespace pd {
namespace {

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
  int vectors;  // rows of logits and of results begin where four elements may be accessed at once
};

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* to, float v) { *to = v; }
__device__ __forceinline__ void put(__nv_bfloat16* to, float v) { *to = __float2bfloat16_rn(v); }

// Four neighbouring logits.
__device__ __forceinline__ void load4(const float* from, float* z) {
  const float4 v = __ldcs(reinterpret_cast<const float4*>(from));
  z[0] = v.x; z[1] = v.y; z[2] = v.z; z[3] = v.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* from, float* z) {
  const uint2 v = __ldcs(reinterpret_cast<const uint2*>(from));
  z[0] = __uint_as_float(v.x << 16); z[1] = __uint_as_float(v.x & 0xffff0000u);
  z[2] = __uint_as_float(v.y << 16); z[3] = __uint_as_float(v.y & 0xffff0000u);
}

// EACH logits per thread.
template <typename In, typename Out, int THREADS, int EACH>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) penalize_logits_kernel(const PenaltyParams p) {
  constexpr int kSlice = THREADS * EACH, kAhead = 8;
  extern __shared__ __align__(16) uint32_t words[];
  griddep_wait();
  griddep_launch_dependents();
  const int row = blockIdx.x / p.slices, first = (blockIdx.x % p.slices) * kSlice;
  const int n = min(kSlice, p.vocab - first);
  const In* src = static_cast<const In*>(p.logits) + (int64_t)row * p.ld + first;
  Out* dst = static_cast<Out*>(p.out) + (int64_t)row * p.ld_out + first;
  // Everything that is read is asked for before anything is waited for, but the history, which waits for its length.
  float r = p.repetition ? p.repetition[row] : 1.f;
  const float f = p.frequency ? p.frequency[row] : 0.f, g = p.presence ? p.presence[row] : 0.f;
  int length = 0;
  if (p.history) length = p.history_len ? p.history_len[row] : p.history_cols;
  const int prompt = p.prompt_len ? p.prompt_len[row] : 0;
  const int mask_row = !p.mask ? -1 : p.mask_row ? p.mask_row[row] : row;
  const int32_t* history = p.history + (int64_t)row * p.ld_history;
  const int32_t* bias_tokens = p.bias_tokens + (int64_t)row * p.bias_cols;
  const int32_t bias_token = (int)threadIdx.x < p.bias_cols ? bias_tokens[threadIdx.x] : -1;
  // this thread's logits: four at a time, THREADS * 4 apart
  float z[EACH];
  auto place = [&](int k) { return (k * THREADS + (int)threadIdx.x) * 4; };
#pragma unroll
  for (int k = 0; k < EACH / 4; ++k) {
    const int j = place(k);
    if (p.vectors && j + 4 <= n) {
      load4(src + j, z + 4 * k);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) z[4 * k + e] = j + e < n ? as_float(src[j + e]) : 0.f;
    }
  }
  if (!(r > 0.f && r <= 3.402823466e38f && 1.f / r <= 3.402823466e38f)) r = 1.f;
  const float inv = 1.f / r;
  length = min(max(length, 0), p.history_cols);
  const bool masked = mask_row >= 0 && mask_row < p.mask_rows;
  const bool counts = length > 0 && (r != 1.f || f != 0.f || g != 0.f);
  const bool changes = counts || p.bias_cols > 0;  // (the same for all threads)
  if (changes) {
    int32_t token[kAhead];
    auto load = [&](int h0) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) token[k] = h0 + k * THREADS < length ? history[h0 + k * THREADS] : -1;
    };
    if (counts) load(threadIdx.x);
#pragma unroll
    for (int k = 0; k < EACH / 4; ++k) *reinterpret_cast<uint4*>(words + place(k)) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (p.bias_cols > 0) {
      auto set_bias = [&](int32_t t, int e) {
        const uint32_t at = (uint32_t)t - (uint32_t)first;
        if (at < (uint32_t)n) atomicMax(words + at, (uint32_t)e + 1u);
      };
      set_bias(bias_token, threadIdx.x);
      for (int e = THREADS + threadIdx.x; e < p.bias_cols; e += THREADS) set_bias(bias_tokens[e], e);
      __syncthreads();
    }
    if (counts) {
      for (int h0 = threadIdx.x; h0 < length; h0 += kAhead * THREADS) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const uint32_t at = (uint32_t)token[k] - (uint32_t)first;
          if (at < (uint32_t)n) {
            if (h0 + k * THREADS >= prompt) atomicAdd(words + at, kOnce);
            else atomicOr(words + at, kOccurs);
          }
        }
        load(h0 + kAhead * THREADS);
      }
      __syncthreads();
    }
  }
  const uint32_t* mask = p.mask + (int64_t)mask_row * p.ld_mask;
  const float* bias_values = p.bias_values + (int64_t)row * p.bias_cols;
#pragma unroll
  for (int k = 0; k < EACH / 4; ++k) {
    const int j = place(k);
    if (j >= n) break;
    float* v = z + 4 * k;
    if (changes) {
      const uint4 w4 = *reinterpret_cast<const uint4*>(words + j);
      if (w4.x | w4.y | w4.z | w4.w) {
        // (few instructions and one branch: in a row with a history most warps come through here; with a division, and a branch for
        // every case, this took 10 us more)
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t times = (w[e] & ~kOccurs) / kOnce;
          v[e] *= w[e] < kOnce ? 1.f : v[e] > 0.f ? inv : r;
          v[e] = times > 0 ? fmaf(-f, (float)times, v[e]) - g : v[e];
        }
        if ((w[0] | w[1] | w[2] | w[3]) & kBiasBits) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (w[e] & kBiasBits) v[e] += bias_values[(w[e] & kBiasBits) - 1];
        }
      }
    }
    if (masked) {
      const uint32_t allowed = __ldg(mask + (first + j) / 32) >> (j % 32);  // (the four lie in one word)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!((allowed >> e) & 1u)) v[e] = -INFINITY;
    }
    if (p.vectors && j + 4 <= n) {
      store_out4(dst, j / 4, make_float4(v[0], v[1], v[2], v[3]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < n) put(dst + j + e, v[e]);
    }
  }
}

template <typename In, typename Out>
pd_status launch(PenaltyParams& p, int64_t rows, cudaStream_t s) {
  // 512 threads, 16384 logits to a slice; 128 and 2048 where that would leave SMs without work.
  const bool narrow = rows * ((p.vocab + 16383) / 16384) < 2 * 148;
  const int slice = narrow ? 2048 : 16384;
  p.slices = (p.vocab + slice - 1) / slice;
  if (rows * p.slices > 0x7fffffff) return PD_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(rows * p.slices));
  const size_t smem = (size_t)slice * 4;
  if (narrow) {
    launch_pdl(penalize_logits_kernel<In, Out, 128, 16>, grid, dim3(128), smem, s, p);
  } else {
    static PerDeviceFlag smem_allowed;
    if (pd_status st = allow_dynamic_smem(penalize_logits_kernel<In, Out, 512, 32>, (int)smem, smem_allowed); st != PD_OK) return st;
    launch_pdl(penalize_logits_kernel<In, Out, 512, 32>, grid, dim3(512), smem, s, p);
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
