// The 8-bit forms of the paged cache: what a stored byte stands for, and where the scale of a block of tokens lies.
// Internal to the library.
#pragma once

#include <cuda_fp16.h>

#include "paged_cache.cuh"

namespace pd {
namespace paged {

// Scales of a cache: [num_pages, heads_kv, page_size / block], one fp32 for the tokens of a block of one head.
struct Scales {
  const float *k, *v;
  int shift;           // log2(block)
  int blocks_per_page;
  int64_t page_stride; // elements from page to page: heads_kv * blocks_per_page
  __device__ __forceinline__ int64_t at(int page, int head, int slot) const {
    return (int64_t)page * page_stride + (int64_t)head * blocks_per_page + (slot >> shift);
  }
};

// Largest magnitude that is written: values are spread over [-top, top].
template <pd_dtype T>
__host__ __device__ constexpr float q8_top() { return T == PD_I8 ? 127.f : 448.f; }

// Two stored values as floats (exact).
template <pd_dtype T>
__device__ __forceinline__ float2 q8_pair_to_float(uint32_t two) {
  if constexpr (T == PD_I8) {
    return make_float2((float)(int8_t)(two & 0xffu), (float)(int8_t)((two >> 8) & 0xffu));
  } else {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
    return __half22float2(*reinterpret_cast<__half2*>(&h));
  }
}

// Two values, already divided by their scale, to the nearest stored ones (ties to even), none beyond the top.
template <pd_dtype T>
__device__ __forceinline__ uint32_t q8_pair_from_float(float a, float b) {
  if constexpr (T == PD_I8) {
    const int x = __float2int_rn(fminf(fmaxf(a, -127.f), 127.f)), y = __float2int_rn(fminf(fmaxf(b, -127.f), 127.f));
    return ((uint32_t)x & 0xffu) | ((uint32_t)y & 0xffu) << 8;
  } else {
    unsigned short two;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(b), "f"(a));
    return two;
  }
}

// The four values of a word as fp16, exactly: bytes 0 and 2 in `even`, 1 and 3 in `odd` (ADJACENT: 0 and 1, 2 and 3).
// int8: 1024 + (x ^ 0x80) has x + 128 in fp16's lowest mantissa bits, so that an and, an xor (one instruction together) and a
// subtraction of 1152 make two values.
template <pd_dtype T, bool ADJACENT>
__device__ __forceinline__ void q8_word_to_half(uint32_t w, uint32_t& even, uint32_t& odd) {
  if constexpr (T == PD_I8) {
    static_assert(!ADJACENT);
    const uint32_t bias = 0x64806480u;  // 1152, twice
    asm("lop3.b32 %0, %2, 0x00ff00ff, %3, 0x6a;\n\t"  // (a & b) ^ c
        "lop3.b32 %1, %4, 0x00ff00ff, %3, 0x6a;"
        : "=r"(even), "=r"(odd) : "r"(w), "r"(bias), "r"(w >> 8));
    asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(even) : "r"(bias));
    asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(odd) : "r"(bias));
  } else {
    if constexpr (!ADJACENT) w = __byte_perm(w, 0, 0x3120);
    asm("{\n\t"
        ".reg .b16 lo, hi;\n\t"
        "mov.b32 {lo, hi}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, lo;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, hi;\n\t"
        "}"
        : "=r"(even), "=r"(odd) : "r"(w));
  }
}

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// ---- host side -----------------------------------------------------------------------
inline bool q8_dtype(pd_dtype t) { return t == PD_I8 || t == PD_E4M3; }
// A power of two that divides the page.
inline bool q8_block_valid(int block, int page_size) { return block > 0 && (block & (block - 1)) == 0 && page_size % block == 0; }
inline Scales make_scales(const pd_cache_scales& s, int heads_kv, int page_size) {
  Scales r{};
  r.k = s.k_scale; r.v = s.v_scale;
  while ((1 << r.shift) < s.block) ++r.shift;
  r.blocks_per_page = page_size >> r.shift;
  r.page_stride = (int64_t)heads_kv * r.blocks_per_page;
  return r;
}

// Tensor map of one cache: {head_dim, page_size, heads_kv, num_pages} bytes, boxes of `box_rows` slots of `box_heads` heads.  What
// is fetched beside a box's rows belongs to other heads, which other CTAs read at other times: promotion to 256 bytes fetched
// twice what rows of 128 need (64 x 1 tokens: 150 us, where the same kernel took 140 without it).
inline bool make_cache_map_q8(CUtensorMap* map, const void* cache, const pd_paged_attention_desc& d, int box_rows, int box_heads) {
  gemm::EncodeTiledFn fn = gemm::encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)d.head_dim, (cuuint64_t)d.page_size, (cuuint64_t)d.heads_kv, (cuuint64_t)d.num_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)d.slot_stride, (cuuint64_t)d.head_stride, (cuuint64_t)d.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)d.head_dim, (cuuint32_t)box_rows, (cuuint32_t)box_heads, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(cache), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            d.head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
            d.head_dim == 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_64B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Launchers (each in its own file).
pd_status launch_chunk_q8(const pd_paged_attention_desc& d, const Params& p, pd_dtype type, const Scales& scales, const void* k_cache,
                          const void* v_cache, cudaStream_t s);
pd_status launch_rows_i8(const pd_paged_attention_desc& d, const Params& p, const Plan& plan, const Scales& scales, const void* k_cache,
                         const void* v_cache, cudaStream_t s);
pd_status launch_rows_e4m3(const pd_paged_attention_desc& d, const Params& p, const Plan& plan, const Scales& scales, const void* k_cache,
                           const void* v_cache, cudaStream_t s);

}  // namespace paged
}  // namespace pd
