// The 8-bit forms of the paged cache: what a stored byte stands for, and where the scale of a block of tokens lies.
// Internal to the library.
#pragma once

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

}  // namespace paged
}  // namespace pd
