// Attention over the paged cache for chunks of tokens, on the tcgen05 tensor cores:
//
//   out[t, h] = sum_j softmax_j(scale * q[t, h] . k[j]) v[j],   j visible from token t's position
//
// Two kernels; the one for a bf16 cache with head_dim 64 is described further down.  In the one for head_dim 128, and for 8-bit
// caches with either, a CTA takes two consecutive
// tiles ("slots") of 128 rows of one cache head (a row is a token and one of the query heads that share the cache head) and
// walks the key tiles of 128 keys that any of them sees; both slots read the same K and V tiles, which halves what comes
// from L2.  While one slot's scores are being exponentiated the other slot's products run.
//
//   warps 0-3, 4-7 : softmax of slot 0 / 1, one thread per row.  For each block of 64 keys: read the row's scores from tensor
//                    memory once, mask them in blocks that are not in view as a whole, and form
//                    p = 2^(s * scale * log2 e - m).  m is a reference that is raised only when a score exceeds it by more
//                    than 2^8 (then the output accumulator and the row sum are rescaled through tensor memory); sums stay
//                    fp32, p is rounded to bf16 and goes back over the scores' columns, where the second product reads it
//                    as its A operand.  At the end the same warps divide by the sum and write the rows.
//   warps 8, 10    : score issuers of slot 0 / 1 (the warp walks the loop, one elected lane issues): S = Q K^T (128 x 64 x D).
//   warps 9, 11    : output issuers: O += P V (128 x D x 64).
//                    (One warp for all four streams spent more time on its waits, 800 clk per block and slot, than the
//                    products take.)
//   warp 12        : producer: looks the pages up and copies K and V tiles by TMA, one box per page, into a ring of four
//                    32 KiB stages, K and V in turn.
//   8-bit caches     : warps 12-15 in its place, which load, convert and write the same tiles (convert_tiles).
//                    (4 chunks of up to 2048 tokens over up to 16384 keys, 32/8 heads of 128, int8: 1137 us a single call, 1238 in long
//                    runs, where the board's power limits the clock; single with the conversions for free 980.  8 prompts of up to 2048,
//                    16 heads of 64, window 1024, e4m3: 186 single, 178 in long runs, 173 with the conversions for free.)
// Tensor memory: per slot two score buffers of 64 columns and an output of 128; that is all of it.  Two
// buffers let the scores of the next block be formed while the current ones are exponentiated: the buffer they take was
// last read by the product of the block before.  (With one buffer of 128 columns the softmax warps of a slot waited half
// their time for two products in a row.)
//
// Values of keys in nobody's view may be anything (stale slots of a page, NaN) and would poison the product with
// probability 0 * NaN: in the tiles that hold such keys the issuers overwrite them with zeros first.
// With `splits` > 1 the key tiles are shared out over that many CTAs, whose partial outputs paged_attention_join joins.
#include <type_traits>

#include "cache_q8.cuh"

namespace pd {
namespace paged {
namespace {

constexpr int kTile = 128;             // keys per tile, and rows per slot
constexpr int kBlock = 64;             // keys per score buffer
constexpr int kSoftmaxWarps = 4;       // per slot
constexpr int kStages = 4;
constexpr int kHalf = kTile * 128;     // 64 columns of a tile: 128 lines of 128 bytes
constexpr float kRaise = 8.f;          // powers of two by which a score may exceed the row's reference
constexpr float kOffset = 7.f;         // powers of two more in P, as fp16: 2^(kRaise + kOffset) is below its largest

// A special-function instruction that keeps its place among the others.
__device__ __forceinline__ float ex2_in_order(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// the lowest n bits, n clamped to [0, 32]
__device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1u; }

// Where keys and values come from.  A bf16 cache: by TMA.
struct TiledCache {
  static constexpr bool kBytes = false, kSwapped = false;
  CUtensorMap k, v;
};
// An 8-bit cache: by plain loads of four warps, which make fp16 of it; Q and P are fp16 then, too.
template <pd_dtype TYPE>
struct ByteCache {
  static constexpr bool kBytes = true, kSwapped = TYPE == PD_I8;  // elements 1 and 2 of every four in the tiles
  static constexpr pd_dtype T = TYPE;
  const uint8_t *k, *v;
  int64_t page_stride, slot_stride, head_stride;
  Scales scales;
};

// Two slots per CTA, one CTA per SM.
template <int HEAD_DIM, typename Cache>
struct WideConfig {
  static constexpr int D = HEAD_DIM, kSlots = 2;
  static constexpr int kProducers = Cache::kBytes ? 4 : 1;  // warps
  static constexpr int kIssuer0 = kSlots * kSoftmaxWarps, kProducer = kIssuer0 + 2 * kSlots;
  static constexpr int kThreads = 32 * (kProducer + kProducers);
  static constexpr int kRows = kSlots * kTile;
  static constexpr int kTensor = kTile * D * 2;  // a Q, K or V tile
  static constexpr int kSmem = kSlots * kTensor + kStages * kTensor + 1024 /*barriers*/ + 1024 /*alignment*/;
  // tensor-memory columns: score buffer b of slot s at 128 s + 64 b (its probabilities over it, two keys to a column), output
  // of slot s behind them
  static constexpr uint32_t kColO = kSlots * kTile, kCols = 512;
};

// The view of one slot: keys [lo, hi) and sinks [0, sink_hi) are seen by some of its rows.
struct SlotView {
  int lo, hi, sink_hi;
  int first_pos, last_pos;
  bool active;
  __device__ __forceinline__ bool needs(int key0) const {
    return active && ((key0 < hi && key0 + kBlock > lo) || key0 < sink_hi);
  }
};

// The output of a warp's 32 rows, one per lane: row (token t of the sequence, head), its reference m, sum l and accumulator (at
// t_o, in units of `unit`, once `any` product has gone into it).  `stage`: shared memory that the warp may use, 32 lines of 128 bytes for every
// 64 columns (its rows of the Q tile, which every product has read by then).  SWAPPED: elements 1 and 2 of every four have
// changed places in the accumulator.
template <int D, bool SWAPPED>
__device__ __forceinline__ void write_rows(const Params& p, const Sequence& seq, int split, int t, int head, bool valid, bool any,
                                           float m, float l, float unit, uint32_t t_o, uint32_t stage) {
  const int lane = threadIdx.x & 31;
  auto place = [](int i) { return SWAPPED && (i % 4 == 1 || i % 4 == 2) ? i ^ 3 : i; };
  tcgen05_fence_after_sync();
  const float inv = l > 0.f ? unit / l : 0.f;  // nothing seen: zeros
  const int64_t at = ((int64_t)split * p.part_tokens + seq.part0 + t) * p.heads_q + head;
  if (p.splits == 1) {
    // through shared memory, so that a store instruction writes whole rows
#pragma unroll
    for (int c = 0; c < D; c += 32) {
      uint32_t o[32];
      if (any) {
        tmem_ld_32x32b_x32(t_o + c, o);
        tmem_ld_wait();
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = any ? pack_bf16(__uint_as_float(o[place(8 * u + 2 * j)]) * inv, __uint_as_float(o[place(8 * u + 2 * j + 1)]) * inv) : 0u;
        const int chunk = c / 8 + u;
        st_shared_v4(stage + (chunk >> 3) * kHalf + (uint32_t)lane * 128u + (uint32_t)(((chunk & 7) ^ (lane & 7)) << 4),
                     make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
    __syncwarp();
    const int64_t out_at = valid ? (int64_t)(seq.q0 + t) * p.ld_out + (int64_t)head * D : -1;  // of this lane's row
    constexpr int kLanes = D / 8;  // 16 bytes each: a row
#pragma unroll 4
    for (int r0 = 0; r0 < 32; r0 += 32 / kLanes) {
      const int r2 = r0 + lane / kLanes, chunk = lane % kLanes;
      const int64_t to = __shfl_sync(0xffffffffu, out_at, r2);
      if (to >= 0) {
        const float4 v = ld_shared_v4_f32(stage + (chunk >> 3) * kHalf + (uint32_t)r2 * 128u + (uint32_t)(((chunk & 7) ^ (r2 & 7)) << 4));
        *reinterpret_cast<float4*>(p.out + to + chunk * 8) = v;
      }
    }
  } else if (any) {
#pragma unroll
    for (int c = 0; c < D; c += 32) {
      uint32_t o[32];
      tmem_ld_32x32b_x32(t_o + c, o);
      tmem_ld_wait();
      if (valid && l > 0.f) {
        float4* dst = reinterpret_cast<float4*>(p.part_o + at * D + c);
#pragma unroll
        for (int u = 0; u < 8; ++u)
          dst[u] = make_float4(__uint_as_float(o[4 * u]) * inv, __uint_as_float(o[place(4 * u + 1)]) * inv,
                               __uint_as_float(o[place(4 * u + 2)]) * inv, __uint_as_float(o[4 * u + 3]) * inv);
      }
    }
  }
  if (valid && p.splits > 1) p.part_lse[at] = l > 0.f ? m + log2f(l) : -INFINITY;
}

// Keys and values of an 8-bit cache into the ring, as fp16: one of four warps, which share every tile, 32 keys each.  A lane has
// 16 elements of a key at a time and loads a whole tile's worth of them ahead, while the tile before is converted.  Keys in
// nobody's view, and ones without a page, become zeros.
//
// A stored byte is exact in fp16.  (Of int8, bytes 0 and 2 of a word become one register and 1 and 3 the other: elements 1 and 2 of
// every four change places, in K as in Q, and in V as in O, where they change back.)  Where the warp's 32 keys share a scale (blocks of 32 tokens and more, usually) that is what goes
// into the product, and the scale goes with the group of 32 keys: to the softmax, which multiplies the group's scores by it, and for
// values adds its logarithm to the exponents and takes it out of the sums.  Where they have several (blocks of 16 tokens and less), the
// elements are multiplied by their scale over the power of two below the largest one that any row sees (as a high and a low fp16, so that
// the product is rounded once, by 2^-11 of it at most), and the power of two goes with the group.  The products take up fp16's range to
// the top, 448 x 128: a scale that is a small part of the group's largest is then off by 2^-31 of that.
//   Instructions per tile and warp: 600 or 1000, where the softmax of the two slots takes 3300 of a scheduler's.  (Elements times their
//   scales in fp32, rounded to bf16, took 1800, and 4 x 2048 tokens over up to 16384 keys 2033 us.)
// factors: of the last four tiles, each 4 scales of keys and 4 logarithms of scales of values, as floats.

// 16 bytes; a load that stays where it is written (the compiler moves a plain one to where its result is used).  Not a non-coherent one: the
// kernel that appends to the cache may have been running when this one started.
__device__ __forceinline__ uint4 load_now(const uint8_t* from) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(from) : "memory");
  return v;
}
__device__ __forceinline__ float load_now(const float* from) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(from));
  return v;
}
template <pd_dtype T>
__device__ __forceinline__ void convert_16(uint4 v, uint32_t (&out)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    q8_word_to_half<T, T != PD_I8>(w[c], out[2 * c], out[2 * c + 1]);
  }
}
constexpr uint32_t kHeadroom = 6;  // powers of two: the largest element times 2^(1 + 6) is in fp16's range
template <int D, typename Cache>
__device__ __forceinline__ void convert_tiles(const Cache& cache, const Params& p, const KeyTiles& kt, int kvh, int b, int begin, int end,
                                              int warp, uint32_t ring, uint32_t bars, uint32_t factors, volatile int* abort_flag) {
  constexpr int kLanes = D / 16, kRowsAtOnce = 32 / kLanes, kSteps = 32 / kRowsAtOnce, kTensor = kTile * D * 2;
  // Eight lanes, whose 16-byte stores go together, have half of two neighbouring lines: the swizzle puts these into different banks.
  const int lane = threadIdx.x & 31, chunk = D == 128 ? (lane & 3) | (lane >> 4) << 2 : lane & 3, in_step = D == 128 ? (lane >> 2) & 3 : lane >> 2;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 32u + 8u * s; };
  uint4 data[2][kSteps];
  // Of the next tile: the page of every step's keys (pages hold eight slots at least, a step's four or eight keys share one),
  // which keys there are, and this lane's key's scales (0 where there is none); of the one behind it this lane's key's page.
  // Pages of 32 slots and more: the group has one page, and the lanes all look that up; blocks of 32 tokens and more: one scale.
  int pages[kSteps], page;
  uint32_t there;
  float scale[2];
  const bool one_page = p.page_size >= 32, one_scale = cache.scales.shift >= 5;
  auto first_key = [&](int i) { return kt.tile_index(i) * kTile + warp * 32; };
  auto look_up = [&](int i) {  // (the entry as it is: to look at it is to wait for it)
    const int entry = i < end ? (first_key(i) + (one_page ? 0 : lane)) >> p.page_shift : p.max_pages;
    page = -1;
    if (entry < p.max_pages) page = __ldg(p.block_table + (int64_t)b * p.max_pages + entry);
  };
  auto locate = [&](int i) {
    if (i >= end) return;
    const int key0 = first_key(i), slot = (key0 + (one_scale ? 0 : lane)) & (p.page_size - 1);
    there = 0xffffffffu;
    if (key0 < kt.lo || key0 + 32 > kt.hi) there = below(kt.hi - key0) & (~below(kt.lo - key0) | below(kt.sink_hi - key0));
    const bool valid = (unsigned)page < (unsigned)p.num_pages;
    if (one_page) {
      pages[0] = page;
      if (!valid) there = 0;
    } else {
      there &= __ballot_sync(0xffffffffu, valid);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) pages[j] = __shfl_sync(0xffffffffu, page, j * kRowsAtOnce);
    }
    const bool mine = one_scale ? there != 0 : (there >> lane) & 1u;
    scale[0] = scale[1] = 0.f;
    if (mine) {
      const int64_t at = cache.scales.at(page, kvh, slot);
      scale[0] = load_now(cache.scales.k + at);
      scale[1] = load_now(cache.scales.v + at);
    }
  };
  const int64_t lane_at = (int64_t)kvh * cache.head_stride + 16 * chunk;
  auto load_data = [&](int i, int kv) {
    if (i >= end) return;
    const int key0 = first_key(i) + in_step;
    const uint8_t* from = (kv == 0 ? cache.k : cache.v) + lane_at;
    if (one_page && there == 0xffffffffu) {
      from += (int64_t)pages[0] * cache.page_stride + (int64_t)(key0 & (p.page_size - 1)) * cache.slot_stride;
#pragma unroll
      for (int j = 0; j < kSteps; ++j, from += kRowsAtOnce * cache.slot_stride) data[kv][j] = load_now(from);
    } else {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const int slot = (key0 + j * kRowsAtOnce) & (p.page_size - 1);
        data[kv][j] = make_uint4(0, 0, 0, 0);
        if ((there >> (j * kRowsAtOnce + in_step)) & 1u)
          data[kv][j] = load_now(from + (int64_t)(one_page ? pages[0] : pages[j]) * cache.page_stride + (int64_t)slot * cache.slot_stride);
      }
    }
  };
  // The factors of tile i's group, and what is left for its keys: this lane's key's scale over the factor, as high and low fp16.
  uint32_t pair[2];
  bool uniform[2], no_values = false;
  auto factor_out = [&](int i) {
    if (i >= end) return;
    float factor[2] = {scale[0], scale[1]};
    uniform[0] = uniform[1] = true;
    if (!one_scale) {
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(scale[kv]));
        uniform[kv] = most == 0;
        const uint32_t exponent = min(max(most >> 23, 1u + kHeadroom), 253u);
        factor[kv] = uniform[kv] ? 0.f : __uint_as_float((exponent - kHeadroom) << 23);
        const float rest = scale[kv] * __uint_as_float((254u + kHeadroom - exponent) << 23);  // below 2^(kHeadroom + 1)
        const __half high = __float2half_rn(rest), low = __float2half_rn(rest - __half2float(high));
        pair[kv] = (uint32_t)__half_as_ushort(high) | (uint32_t)__half_as_ushort(low) << 16;
      }
    }
    no_values = factor[1] == 0.f;  // a scale of zero: zeros, whatever is stored
    if (lane == 0) {
      const uint32_t to = factors + 32u * ((i - begin) & 3) + 4u * warp;
      st_shared_f32(to, factor[0]);
      st_shared_f32(to + 16u, __log2f(factor[1]));
    }
  };
  if (p.withhold_loads || begin >= end) return;
  look_up(begin);
  locate(begin);
  look_up(begin + 1);
  load_data(begin, 0);
  load_data(begin, 1);
  factor_out(begin);
  locate(begin + 1);
  look_up(begin + 2);
  int n = 0;
  for (int i = begin; i < end; ++i) {
#pragma unroll
    for (int kv = 0; kv < 2; ++kv, ++n) {
      const int stage = n % kStages;
      if (!mbar_wait_warp(empty(stage), ((n / kStages) & 1u) ^ 1u, abort_flag, p.status, kTimeoutChunkProducer, p.wait_limit_ns)) return;
      auto store = [&](int j, const uint32_t (&out)[8]) {
        const int r = warp * 32 + j * kRowsAtOnce + in_step;
        const uint32_t row = ring + stage * kTensor + (chunk >> 2) * kHalf + (uint32_t)r * 128u;
#pragma unroll
        for (int c = 0; c < 2; ++c)
          st_shared_v4(row + (uint32_t)((((2 * chunk + c) & 7) ^ (r & 7)) << 4), make_uint4(out[4 * c], out[4 * c + 1], out[4 * c + 2], out[4 * c + 3]));
      };
      if (uniform[kv]) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          uint32_t out[8];
          convert_16<Cache::T>(kv == 1 && no_values ? make_uint4(0, 0, 0, 0) : data[kv][j], out);
          store(j, out);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          uint32_t out[8];
          convert_16<Cache::T>(data[kv][j], out);
          const uint32_t mine = __shfl_sync(0xffffffffu, pair[kv], j * kRowsAtOnce + in_step);
          const uint32_t high = __byte_perm(mine, 0, 0x1010), low = __byte_perm(mine, 0, 0x3232);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            uint32_t t;
            asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(t) : "r"(out[c]), "r"(low));
            asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(out[c]) : "r"(out[c]), "r"(high), "r"(t));
          }
          store(j, out);
        }
      }
      load_data(i + 1, kv);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(full(stage));
    }
    // What needs an answer from the shared-memory pipe (it works through the stores above first, between the products' reads)
    // comes once a tile, here.
    factor_out(i + 1);
    locate(i + 2);
    look_up(i + 3);
  }
}

template <int D, typename Cache>
__global__ void __launch_bounds__(WideConfig<D, Cache>::kThreads, 1)
paged_attention_chunk_kernel(const __grid_constant__ Cache cache, const Params p) {
  using C = WideConfig<D, Cache>;
  constexpr int kSlots = C::kSlots, kIssuer0 = C::kIssuer0, kProducer = C::kProducer;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = base, ring = sQ + kSlots * C::kTensor, bars = ring + kStages * C::kTensor;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 32u + 8u * s; };
  auto q_full = [&](int s) { return bars + 64u + 8u * s; };
  auto s_full = [&](int s, int b) { return bars + 80u + 16u * s + 8u * b; };
  auto p_full = [&](int s, int b) { return bars + 112u + 16u * s + 8u * b; };
  auto o_full = [&](int s, int b) { return bars + 144u + 16u * s + 8u * b; };  // the product that read buffer b has completed
  auto drained = [&](int w) { return bars + 176u + 8u * w; };  // of the four issuers
  const uint32_t factors = bars + 256u;                        // 8-bit caches: of four tiles
  uint8_t* ctrl = smem_raw + (bars - smem_u32(smem_raw)) + 512;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(full(s), C::kProducers); mbar_init(empty(s), kSlots); }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(q_full(s), kSoftmaxWarps);
      for (int b = 0; b < 2; ++b) { mbar_init(o_full(s, b), 1); mbar_init(s_full(s, b), 1); mbar_init(p_full(s, b), kSoftmaxWarps); }
    }
    for (int w = 0; w < 2 * kSlots; ++w) mbar_init(drained(w), 1);
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == kProducer) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), C::kCols);
    tmem_relinquish_alloc_permit();
    if constexpr (!Cache::kBytes) {
      if (lane == 0) { prefetch_tensormap(&cache.k); prefetch_tensormap(&cache.v); }
    }
  }
  tcgen05_fence_before_sync();
  __syncthreads();
  tcgen05_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  griddep_wait();
  griddep_launch_dependents();

  const int split = blockIdx.x % p.splits;
  const int tiles = gridDim.x / p.splits;
  const int tile = tiles - 1 - blockIdx.x / p.splits;  // the last rows see the most keys: they go first
  const int kvh = blockIdx.y, b = blockIdx.z;
  const Sequence seq = load_sequence(p, b);
  const int all_rows = seq.n * p.group, row0 = tile * C::kRows;
  if (row0 < all_rows) {
    const int last_row = min(row0 + C::kRows, all_rows) - 1;
    const KeyTiles kt = key_tiles(p, seq.pos0 + row0 / p.group, seq.pos0 + last_row / p.group, seq.length, kTile);
    int begin, end;
    split_range(p, kt.n, split, begin, end);
    const int blocks = 2 * (end - begin);
    auto block_key = [&](int b) { return kt.tile_index(begin + (b >> 1)) * kTile + (b & 1) * kBlock; };
    auto slot_view = [&](int s) {
      SlotView v;
      const int r0 = row0 + s * kTile;
      v.active = r0 < all_rows;
      v.first_pos = seq.pos0 + r0 / p.group;
      v.last_pos = seq.pos0 + (min(r0 + kTile, all_rows) - 1) / p.group;
      const KeyTiles t = key_tiles(p, v.first_pos, v.last_pos, seq.length, kTile);
      v.lo = t.lo; v.hi = t.hi; v.sink_hi = t.sink_hi;
      return v;
    };

    if (warp < kIssuer0) {
      // ------------------------------------------------------------------- softmax
      const int s = warp >> 2, quarter = warp & 3;
      const int r = quarter * 32 + lane, row = row0 + s * kTile + r;
      const SlotView view = slot_view(s);
      const bool valid = row < all_rows;
      const int t = valid ? row / p.group : 0, head = kvh * p.group + (valid ? row % p.group : 0);
      const int pos = seq.pos0 + t;
      float row_scale = p.scale_log2e;
      if (view.active) {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(seq.q0 + t) * p.ld_q + (int64_t)head * D);
        const uint32_t dst = sQ + s * C::kTensor + (uint32_t)r * 128u;
        float up = 1.f;
        if constexpr (Cache::kBytes) {
          // fp16: the row's largest magnitude is taken to [2^14, 2^15) by a power of two, which the scores are divided by again
          uint32_t most = 0;
#pragma unroll
          for (int c = 0; c < D / 8; ++c) {
            const uint4 v = valid ? src[c] : make_uint4(0, 0, 0, 0);
            most = max(most, max(max((v.x << 16) & 0x7fffffffu, v.x & 0x7fff0000u), max((v.y << 16) & 0x7fffffffu, v.y & 0x7fff0000u)));
            most = max(most, max(max((v.z << 16) & 0x7fffffffu, v.z & 0x7fff0000u), max((v.w << 16) & 0x7fffffffu, v.w & 0x7fff0000u)));
          }
          const int shift = min(max(14 + 127 - (int)(most >> 23), -126), 126);
          up = __uint_as_float((uint32_t)(127 + shift) << 23);
          row_scale *= __uint_as_float((uint32_t)(127 - shift) << 23);
        }
#pragma unroll
        for (int c0 = 0; c0 < D / 8; c0 += 8) {
          uint4 raw[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) raw[c] = valid ? src[c0 + c] : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            uint4 v = raw[c];
            if constexpr (Cache::kBytes) {
              auto low = [&](uint32_t two) { return __uint_as_float(two << 16) * up; };
              auto high = [&](uint32_t two) { return __uint_as_float(two & 0xffff0000u) * up; };
              if constexpr (Cache::kSwapped)
                v = make_uint4(pack_half(low(v.x), low(v.y)), pack_half(high(v.x), high(v.y)), pack_half(low(v.z), low(v.w)), pack_half(high(v.z), high(v.w)));
              else
                v = make_uint4(pack_half(low(v.x), high(v.x)), pack_half(low(v.y), high(v.y)), pack_half(low(v.z), high(v.z)), pack_half(low(v.w), high(v.w)));
            }
            st_shared_v4(dst + (c0 >> 3) * kHalf + (uint32_t)((c ^ (r & 7)) << 4), v);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full(s));
      }
      const uint32_t t_lane = tmem + ((uint32_t)(quarter * 32) << 16);
      const uint32_t t_o = t_lane + C::kColO + s * D;
      float m = -INFINITY, l = 0.f;
      // 8-bit caches: O is in units of 2^unit, more than the largest scale of values that the row has seen so far; P carries kOffset powers of
      // two more, so that what fp16 loses of small exponentials is below 2^-30 of the largest
      float unit = -1e30f;
      uint32_t done = 0;  // blocks of this slot
      bool ok = true;
      for (int b = 0; b < blocks; ++b) {
        const int key0 = block_key(b);
        if (!view.needs(key0)) continue;
        const int buf = done & 1;
        const uint32_t t_s = t_lane + s * kTile + buf * kBlock;
        if (!mbar_wait_warp(s_full(s, buf), (done >> 1) & 1u, abort_flag, p.status, kTimeoutChunkSoftmax, p.wait_limit_ns)) { ok = false; break; }
        tcgen05_fence_after_sync();
        uint32_t x[2][32];
        tmem_ld_32x32b_x32(t_s, x[0]);
        tmem_ld_32x32b_x32(t_s + 32, x[1]);
        tmem_ld_wait();
        const bool whole = key0 + kBlock - 1 <= view.first_pos && key0 + kBlock <= seq.length &&
                           (p.window == 0 || key0 > view.last_pos - p.window || key0 + kBlock <= p.sinks);
        if (!whole) {
          // columns [low, high) and [0, sink) of the block are in this row's view
          const int high = min(pos + 1, seq.length) - key0;
          const int low = p.window > 0 ? pos - p.window + 1 - key0 : 0;
          const int sink = p.window > 0 ? p.sinks - key0 : 0;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint32_t seen = below(high - 32 * c) & (~below(low - 32 * c) | below(sink - 32 * c));
            if (__any_sync(0xffffffffu, seen != 0xffffffffu)) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!((seen >> j) & 1u)) x[c][j] = 0xff800000u;  // -inf
            }
          }
        }
        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < 32; j += 4)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            mx4[c] = max3(mx4[c], __uint_as_float(x[c >> 1][j + 2 * (c & 1)]), __uint_as_float(x[c >> 1][j + 2 * (c & 1) + 1]));
        // of either half of the block: the scale of its scores, and what its exponents get beside them
        float scale[2] = {p.scale_log2e, p.scale_log2e}, shift[2] = {0.f, 0.f}, mx;
        bool grown = false;
        if constexpr (Cache::kBytes) {
          const uint32_t at = factors + 32u * ((b >> 1) & 3) + 8u * (b & 1);
          const float2 k = ld_shared_v2_f32(at), v = ld_shared_v2_f32(at + 16u);
          scale[0] = fmaxf(k.x * row_scale, 1.17549435e-38f);  // (-inf times it stays -inf)
          scale[1] = fmaxf(k.y * row_scale, 1.17549435e-38f);
          mx = fmaxf(fmaxf(mx4[0], mx4[1]) * scale[0], fmaxf(mx4[2], mx4[3]) * scale[1]);
          // (a half that this row sees nothing of does not count)
          shift[0] = fmaxf(mx4[0], mx4[1]) > -INFINITY ? v.x : -INFINITY;
          shift[1] = fmaxf(mx4[2], mx4[3]) > -INFINITY ? v.y : -INFINITY;
          grown = fmaxf(shift[0], shift[1]) > unit;
        } else {
          mx = fmaxf(max3(mx4[0], mx4[1], mx4[2]), mx4[3]) * p.scale_log2e;
        }
        const bool raise = mx > m + kRaise;  // also the first finite score of a row (m = -inf)
        if (__any_sync(0xffffffffu, raise || grown)) {
          float alpha = raise ? ex2(m - mx) : 1.f;
          if (raise) m = mx;
          l *= alpha;
          if (grown) {
            const float larger = ceilf(fmaxf(shift[0], shift[1])) + 1.f;
            alpha *= ex2(unit - larger);
            unit = larger;
          }
          if (done > 0) {
            // every product into O so far has to be through with it; the one before last is, or these scores would not be here
            if (!mbar_wait_warp(o_full(s, buf ^ 1), ((done - 1) >> 1) & 1u, abort_flag, p.status, kTimeoutChunkSoftmax, p.wait_limit_ns)) { ok = false; break; }
            tcgen05_fence_after_sync();
#pragma unroll 1
            for (int c = 0; c < D; c += 8) {
              uint32_t o[8];
              tmem_ld_32x32b_x8(t_o + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
              tmem_st_32x32b_x8(t_o + c, o);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        uint64_t scale2[2], nref2[2], sum2[2][2] = {{0, 0}, {0, 0}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // (a half without values to speak of is kept 100 powers of two below the unit, where the exponentials are still there to be added up)
          if constexpr (Cache::kBytes) shift[h] = fmaxf(shift[h] - unit, -100.f);
          const float add = Cache::kBytes ? kOffset + shift[h] - ref : -ref;
          scale2[h] = pack_f32x2(scale[h], scale[h]);
          nref2[h] = pack_f32x2(add, add);
        }
        uint32_t pk[32];
        // Groups of sixteen, each group's sums and packing behind the next one's exponentials, in this order: left to the
        // compiler, the special-function unit stood idle between them (894 against 867 us for 4 x 2048 tokens; 790 with no
        // exponentials at all).
        auto scale_group = [&](int g) {
#pragma unroll
          for (int j = 16 * g; j < 16 * g + 16; j += 2) {
            uint32_t(&v)[32] = x[j >> 5];
            float a0, a1;
            unpack_f32x2(fma_f32x2(pack_b32x2(v[j & 31], v[(j & 31) + 1]), scale2[j >> 5], nref2[j >> 5]), a0, a1);
            v[j & 31] = __float_as_uint(a0);
            v[(j & 31) + 1] = __float_as_uint(a1);
          }
#pragma unroll
          for (int j = 16 * g; j < 16 * g + 16; ++j)
            x[j >> 5][j & 31] = __float_as_uint(ex2_in_order(__uint_as_float(x[j >> 5][j & 31])));
        };
        auto pack_group = [&](int g) {
#pragma unroll
          for (int j = 16 * g; j < 16 * g + 16; j += 2) {
            uint32_t(&v)[32] = x[j >> 5];
            uint64_t& sum = sum2[Cache::kBytes ? j >> 5 : 0][(j >> 1) & 1];
            sum = add_f32x2(sum, pack_b32x2(v[j & 31], v[(j & 31) + 1]));
            if constexpr (Cache::kBytes) {
              pk[j / 2] = pack_half(__uint_as_float(v[j & 31]), __uint_as_float(v[(j & 31) + 1]));
            } else {
              pk[j / 2] = pack_bf16(__uint_as_float(v[j & 31]), __uint_as_float(v[(j & 31) + 1]));
            }
          }
        };
        scale_group(0);
        scale_group(1);
        pack_group(0);
        scale_group(2);
        pack_group(1);
        scale_group(3);
        pack_group(2);
        pack_group(3);
        tmem_st_32x32b_x32(t_s, pk);
        float s0, s1;
        unpack_f32x2(add_f32x2(sum2[0][0], sum2[0][1]), s0, s1);
        if constexpr (Cache::kBytes) {
          float s2, s3;
          unpack_f32x2(add_f32x2(sum2[1][0], sum2[1][1]), s2, s3);
          l += (s0 + s1) * ex2(-shift[0]) + (s2 + s3) * ex2(-shift[1]);
        } else {
          l += s0 + s1;
        }
        tmem_st_wait();
        tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(s, buf));
        ++done;
      }
      // ---- the row's output
      if (ok && done > 0) ok = mbar_wait_warp(o_full(s, (done - 1) & 1), ((done - 1) >> 1) & 1u, abort_flag, p.status, kTimeoutChunkSoftmax, p.wait_limit_ns);
      if (ok && view.active && *abort_flag == 0) {
        write_rows<D, Cache::kSwapped>(p, seq, split, t, head, valid, done > 0, Cache::kBytes ? m - kOffset : m, l, Cache::kBytes ? ex2(unit) : 1.f, t_o,
                      sQ + s * C::kTensor + (uint32_t)(quarter * 32) * 128u);
      }
    } else if (warp >= kProducer) {
      if constexpr (Cache::kBytes) {
        // ---------------------------------------------------------------- converters
        convert_tiles<D>(cache, p, kt, kvh, b, begin, end, warp - kProducer, ring, bars, factors, abort_flag);
      } else {
        // ------------------------------------------------------------------ producer
        const int box = min(p.page_size, kTile);
        const int per_tile = kTile / box, per_batch = 32 / per_tile;
        int page = 0, n = 0;  // n: ring slots requested so far
        bool ok = !p.withhold_loads;
        for (int i = begin; i < end && ok; ++i) {
          const int in_batch = (i - begin) % per_batch;
          if (in_batch == 0) {
            const int ti = i + lane / per_tile;
            page = ti < end ? page_of(p, b, kt.tile_index(ti) * kTile + (lane % per_tile) * box) : 0;
          }
          const int slot = (kt.tile_index(i) * kTile) & (p.page_size - 1);
          for (int kv = 0; kv < 2; ++kv, ++n) {
            const int stage = n % kStages;
            if (!mbar_wait_warp(empty(stage), ((n / kStages) & 1u) ^ 1u, abort_flag, p.status, kTimeoutChunkProducer, p.wait_limit_ns)) { ok = false; break; }
            if (elect_one()) mbar_arrive_expect_tx(full(stage), C::kTensor);
            __syncwarp();
            for (int j = 0; j < per_tile; ++j) {
              const int pg = __shfl_sync(0xffffffffu, page, in_batch * per_tile + j);
              if (elect_one()) {
#pragma unroll
                for (int h = 0; h < D / 64; ++h)
                  tma_load_4d(ring + stage * C::kTensor + h * kHalf + j * box * 128, kv == 0 ? &cache.k : &cache.v, full(stage),
                              h * 64, slot, kvh, pg);
              }
              __syncwarp();
            }
          }
        }
        // Leave no copy in flight, whichever warp gives up: the last request of every stage gets a short time to land.
        volatile int never = 0;
        for (int back = 1; back <= kStages && back <= n; ++back)
          mbar_wait(full((n - back) % kStages), ((n - back) / kStages) & 1u, &never, nullptr, 0, 20000000ull);
      }
    } else {
      // --------------------------------------------------------------- MMA issuers
      const int s = (warp - kIssuer0) >> 1;
      const SlotView view = slot_view(s);
      uint32_t k = 0;  // products issued so far
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        ok = ok && mbar_wait_warp(bar, parity & 1u, abort_flag, p.status, kTimeoutChunkMma, p.wait_limit_ns);
        return ok;
      };
      constexpr uint64_t kBlockStep = (kBlock * 128) >> 4;  // descriptor step from a tile's first block to its second
      if (((warp - kIssuer0) & 1) == 0) {
        // ---- scores; K tile t is in ring slot 2 t
        constexpr uint32_t idesc = Cache::kBytes ? make_idesc_f16(kTile, kBlock, false, false) : make_idesc_bf16(kTile, kBlock, false, false);
        const uint64_t q_desc = make_smem_desc(sQ + s * C::kTensor, 0, 1024);
        if (view.active) wait(q_full(s), 0);
        for (int b = 0; b < blocks && ok; ++b) {
          const int n = b & ~1, stage = n % kStages;
          if ((b & 1) == 0 && !wait(full(stage), n / kStages)) break;
          if (view.needs(block_key(b))) {
            const uint32_t buf = k & 1u;
            // the buffer holds the probabilities of the block before last: the product that reads them must have completed
            if (k >= 2 && !wait(o_full(s, buf), (k >> 1) - 1)) break;
            tcgen05_fence_after_sync();
            const uint64_t k_desc = make_smem_desc(ring + stage * C::kTensor, 0, 1024) + (b & 1) * kBlockStep;
            if (elect_one()) {
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks) {
                const uint64_t step = (uint64_t)((ks >> 2) * (kHalf >> 4) + (ks & 3) * 2);
                mma_bf16_ss(tmem + s * kTile + buf * kBlock, q_desc + step, k_desc + step, idesc, ks != 0 ? 1u : 0u);
              }
              mma_commit(s_full(s, buf));
            }
            __syncwarp();
            ++k;
          }
          if ((b & 1) && elect_one()) mma_commit(empty(stage));  // both slots' issuers arrive, in need of the tile or not
          __syncwarp();
        }
      } else {
        // ---- output; V tile t is in ring slot 2 t + 1
        constexpr uint32_t idesc = Cache::kBytes ? make_idesc_f16(kTile, D, false, true) : make_idesc_bf16(kTile, D, false, true);  // V is MN-major
        for (int b = 0; b < blocks && ok; ++b) {
          const int n = b | 1, stage = n % kStages;
          const int key0 = block_key(b);
          if ((b & 1) == 0) {
            if (!wait(full(stage), n / kStages)) break;
            if (!Cache::kBytes && (view.needs(key0) || view.needs(key0 + kBlock)) &&
                (key0 + kTile > kt.hi || (key0 < kt.lo && key0 + kTile > kt.sink_hi))) {
              // values of keys in nobody's view: zeros (both slots' issuers write the same; neither's product reads the
              // tile before its own are in; the converters of an 8-bit cache have left zeros there)
              const uint32_t v_tile = ring + stage * C::kTensor;
              for (int r = lane; r < kTile; r += 32) {
                const int key = key0 + r;
                if (!((key < kt.hi && key >= kt.lo) || key < kt.sink_hi)) {
#pragma unroll
                  for (int c = 0; c < D / 8; ++c)
                    st_shared_v4(v_tile + (c >> 3) * kHalf + r * 128 + (c & 7) * 16, make_uint4(0, 0, 0, 0));
                }
              }
              fence_proxy_async_smem();
              __syncwarp();
            }
          }
          if (view.needs(key0)) {
            const uint32_t buf = k & 1u;
            if (!wait(p_full(s, buf), k >> 1)) break;
            tcgen05_fence_after_sync();
            const uint64_t v_desc = make_smem_desc(ring + stage * C::kTensor, kHalf, 1024) + (b & 1) * kBlockStep;
            if (elect_one()) {
#pragma unroll
              for (int ks = 0; ks < kBlock / 16; ++ks)
                mma_bf16_ts(tmem + C::kColO + s * D, tmem + s * kTile + buf * kBlock + 8 * ks,
                            v_desc + (uint64_t)(ks * ((16 * 128) >> 4)), idesc, (k == 0 && ks == 0) ? 0u : 1u);
              mma_commit(o_full(s, buf));
            }
            __syncwarp();
            ++k;
          }
          if ((b & 1) && elect_one()) mma_commit(empty(stage));
          __syncwarp();
        }
      }
      // Products in flight still read shared and tensor memory: whichever warp gives up, they get a short time to end.
      if (elect_one()) mma_commit(drained(warp - kIssuer0));
      __syncwarp();
      volatile int never = 0;
      mbar_wait(drained(warp - kIssuer0), 0, &never, nullptr, 0, 20000000ull);
    }
  }

  // ------------------------------------------------------------------------ teardown
  __syncwarp();
  tcgen05_fence_before_sync();
  __syncthreads();
  if (warp == kProducer) {
    tcgen05_fence_after_sync();
    tmem_dealloc(tmem, C::kCols);
  }
}

// ---- head_dim 64 -----------------------------------------------------------------------
// A block of 128 x 64 scores costs twice as much of the special-function unit (512 clk) as of the tensor pipe.  What bounds the
// kernel is neither, but the serial chain of a CTA (keys, scores, softmax, product, the next scores over the same buffer): of
// the 240 us below 202 remain without any exponential, and 181 without any softmax arithmetic.  One slot per CTA and four
// CTAs per SM let the chains cover each other, and each other's start and end (they weigh where a window keeps the walk
// short).  That leaves a CTA 128 columns of tensor memory, one
// buffer of scores and the output, and 96 registers a thread, so that the scores are read once for the maximum, and the second
// half of a row once more for the exponentials, and a ring of two slots.  One warp issues both products and requests a slot
// again once the product that read it has completed.
//   8 prompts of up to 4096 tokens, 16 heads, window 1024: 240 us, 62 to 70 % of the special-function unit's rate on long walks.
//   Two CTAs per SM with two buffers and the roles of the other kernel: 270.  Blocks of 32 keys in two buffers, four CTAs: 270
//   (a product of 128 x 32 x 16 takes 40 clk, its 128 x 16 operand being read from shared memory at 128 bytes/clk; one of
//   128 x 64 x 16 48, where the arithmetic needs 16 and 32).  Exponentials in another order, or the product split in halves to
//   start earlier: no change.
struct NarrowConfig {
  static constexpr int D = 64, kStages = 2, kCtasPerSm = 4;
  static constexpr int kThreads = 32 * (kSoftmaxWarps + 1);
  static constexpr int kQ = kTile * D * 2, kTensor = kBlock * D * 2;  // bytes of the Q tile, of a block of K or V
  static constexpr int kSmem = kQ + kStages * 2 * kTensor + 1024 /*barriers*/ + 1024 /*alignment*/;
  static constexpr uint32_t kColO = 64, kCols = 128;  // scores, the output behind them
  static_assert(kCtasPerSm * (kSmem + 1024) <= 228 * 1024 && kCtasPerSm * kCols <= 512);
};

__global__ void __launch_bounds__(NarrowConfig::kThreads, NarrowConfig::kCtasPerSm)
paged_attention_chunk_narrow_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                                    const Params p) {
  using C = NarrowConfig;
  constexpr int D = C::D, kStages = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = base, ring = sQ + C::kQ, bars = ring + kStages * 2 * C::kTensor;
  auto full = [&](int s) { return bars + 8u * s; };
  const uint32_t s_full = bars + 32u, p_full = bars + 48u, o_full = bars + 64u, q_full = bars + 80u, drained = bars + 88u;
  uint8_t* ctrl = smem_raw + (bars - smem_u32(smem_raw)) + 512;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(full(s), 1);
    mbar_init(s_full, 1);
    mbar_init(p_full, kSoftmaxWarps);
    mbar_init(o_full, 1);
    mbar_init(q_full, kSoftmaxWarps);
    mbar_init(drained, 1);
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == kSoftmaxWarps) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), C::kCols);
    tmem_relinquish_alloc_permit();
    if (lane == 0) { prefetch_tensormap(&tmap_k); prefetch_tensormap(&tmap_v); }
  }
  tcgen05_fence_before_sync();
  __syncthreads();
  tcgen05_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  griddep_wait();
  griddep_launch_dependents();

  const int split = blockIdx.x % p.splits;
  const int tiles = gridDim.x / p.splits;
  const int tile = tiles - 1 - blockIdx.x / p.splits;  // the last rows see the most keys: they go first
  const int kvh = blockIdx.y, b = blockIdx.z;
  const Sequence seq = load_sequence(p, b);
  const int all_rows = seq.n * p.group, row0 = tile * kTile;
  if (row0 < all_rows) {
    const int first_pos = seq.pos0 + row0 / p.group, last_pos = seq.pos0 + (min(row0 + kTile, all_rows) - 1) / p.group;
    const KeyTiles kt = key_tiles(p, first_pos, last_pos, seq.length, kBlock);
    int begin, end;
    split_range(p, kt.n, split, begin, end);
    const int blocks = end - begin;

    if (warp < kSoftmaxWarps) {
      // ------------------------------------------------------------------- softmax
      const int r = warp * 32 + lane, row = row0 + r;
      const bool valid = row < all_rows;
      const int t = valid ? row / p.group : 0, head = kvh * p.group + (valid ? row % p.group : 0);
      const int pos = seq.pos0 + t;
      const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(seq.q0 + t) * p.ld_q + (int64_t)head * D);
      uint4 raw[D / 8];
#pragma unroll
      for (int c = 0; c < D / 8; ++c) raw[c] = valid ? src[c] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int c = 0; c < D / 8; ++c) st_shared_v4(sQ + (uint32_t)r * 128u + (uint32_t)((c ^ (r & 7)) << 4), raw[c]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
      const uint32_t t_lane = tmem + ((uint32_t)(warp * 32) << 16), t_o = t_lane + C::kColO;
      const uint64_t scale2 = pack_f32x2(p.scale_log2e, p.scale_log2e);
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      for (int i = 0; i < blocks; ++i) {
        const int key0 = kt.tile_index(begin + i) * kBlock;
        if (!mbar_wait_warp(s_full, i & 1u, abort_flag, p.status, kTimeoutChunkSoftmax, p.wait_limit_ns)) { ok = false; break; }
        tcgen05_fence_after_sync();
        uint32_t x[32], x1[32];
        tmem_ld_32x32b_x32(t_lane, x);
        tmem_ld_32x32b_x32(t_lane + 32, x1);
        tmem_ld_wait();
        const bool whole = key0 + kBlock - 1 <= first_pos && key0 + kBlock <= seq.length &&
                           (p.window == 0 || key0 > last_pos - p.window || key0 + kBlock <= p.sinks);
        uint32_t seen[2] = {0xffffffffu, 0xffffffffu};
        auto mask = [&](uint32_t (&v)[32], uint32_t bits) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (!((bits >> j) & 1u)) v[j] = 0xff800000u;  // -inf
        };
        if (!whole) {
          // columns [low, high) and [0, sink) of the block are in this row's view
          const int high = min(pos + 1, seq.length) - key0;
          const int low = p.window > 0 ? pos - p.window + 1 - key0 : 0;
          const int sink = p.window > 0 ? p.sinks - key0 : 0;
          seen[0] = below(high) & (~below(low) | below(sink));
          seen[1] = below(high - 32) & (~below(low - 32) | below(sink - 32));
          mask(x, seen[0]);
          mask(x1, seen[1]);
        }
        float mx2[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < 32; j += 4)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            mx2[c] = max3(mx2[c], __uint_as_float(x[j + 2 * c]), __uint_as_float(x[j + 2 * c + 1]));
            mx2[c] = max3(mx2[c], __uint_as_float(x1[j + 2 * c]), __uint_as_float(x1[j + 2 * c + 1]));
          }
        const float mx = fmaxf(mx2[0], mx2[1]) * p.scale_log2e;
        const bool raise = mx > m + kRaise;  // also the first finite score of a row (m = -inf)
        if (__any_sync(0xffffffffu, raise)) {
          const float alpha = raise ? ex2(m - mx) : 1.f;
          if (raise) m = mx;
          l *= alpha;
          if (i > 0) {
            // (the products into O so far are through with it, or these scores would not be here)
#pragma unroll 1
            for (int c = 0; c < D; c += 8) {
              uint32_t o[8];
              tmem_ld_32x32b_x8(t_o + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
              tmem_st_32x32b_x8(t_o + c, o);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        const uint64_t nref2 = pack_f32x2(-ref, -ref);
        uint64_t sum2[2] = {0, 0};
        auto exponentials = [&](uint32_t to) {  // of the 32 scores in x: summed, rounded, and stored over columns that have been read
          uint32_t pk[16];
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            float a0, a1;
            unpack_f32x2(fma_f32x2(pack_b32x2(x[j], x[j + 1]), scale2, nref2), a0, a1);
            a0 = ex2(a0);
            a1 = ex2(a1);
            sum2[(j >> 1) & 1] = add_f32x2(sum2[(j >> 1) & 1], pack_f32x2(a0, a1));
            pk[j / 2] = pack_bf16(a0, a1);
          }
          tmem_st_32x32b_x16(to, pk);
        };
        exponentials(t_lane);
        tmem_ld_32x32b_x32(t_lane + 32, x);
        tmem_ld_wait();
        if (!whole) mask(x, seen[1]);
        exponentials(t_lane + 16);
        float s0, s1;
        unpack_f32x2(add_f32x2(sum2[0], sum2[1]), s0, s1);
        l += s0 + s1;
        tmem_st_wait();
        tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full);
      }
      if (ok && blocks > 0)
        ok = mbar_wait_warp(o_full, (blocks - 1) & 1u, abort_flag, p.status, kTimeoutChunkSoftmax, p.wait_limit_ns);
      if (ok && *abort_flag == 0)
        write_rows<D, false>(p, seq, split, t, head, valid, blocks > 0, m, l, 1.f, t_o, sQ + (uint32_t)(warp * 32) * 128u);
    } else {
      // ------------------------------------------- producer and issuer of both products
      const int box = min(p.page_size, kBlock);
      const int per_tile = kBlock / box, per_batch = 32 / per_tile;
      int page = 0;
      // K and V of block i, into ring slot i % kStages
      auto slot_at = [&](int i) { return ring + (uint32_t)(i % kStages) * (2 * C::kTensor); };
      auto request = [&](int i) {
        const int in_batch = i % per_batch;
        if (in_batch == 0) {  // the lanes hold the pages of the next `per_batch` blocks
          const int ti = i + lane / per_tile;
          page = ti < blocks ? page_of(p, b, kt.tile_index(begin + ti) * kBlock + (lane % per_tile) * box) : 0;
        }
        const int first = (kt.tile_index(begin + i) * kBlock) & (p.page_size - 1);
        const uint32_t bar = full(i % kStages);
        if (elect_one()) mbar_arrive_expect_tx(bar, 2 * C::kTensor);
        __syncwarp();
        for (int j = 0; j < per_tile; ++j) {
          const int pg = __shfl_sync(0xffffffffu, page, in_batch * per_tile + j);
          if (elect_one()) {
            tma_load_4d(slot_at(i) + j * box * 128, &tmap_k, bar, 0, first, kvh, pg);
            tma_load_4d(slot_at(i) + C::kTensor + j * box * 128, &tmap_v, bar, 0, first, kvh, pg);
          }
          __syncwarp();
        }
      };
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        ok = ok && mbar_wait_warp(bar, parity & 1u, abort_flag, p.status, kTimeoutChunkMma, p.wait_limit_ns);
        return ok;
      };
      constexpr uint32_t s_idesc = make_idesc_bf16(kTile, kBlock, false, false);
      constexpr uint32_t o_idesc = make_idesc_bf16(kTile, D, false, true);  // V is MN-major
      const uint64_t q_desc = make_smem_desc(sQ, 0, 1024);
      // scores of block i, once its keys are there (and its buffer is free)
      auto scores = [&](int i) {
        if (!wait(full(i % kStages), i / kStages)) return;
        tcgen05_fence_after_sync();
        const uint64_t k_desc = make_smem_desc(slot_at(i), 0, 1024);
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
            mma_bf16_ss(tmem, q_desc + 2 * ks, k_desc + 2 * ks, s_idesc, ks != 0 ? 1u : 0u);
          mma_commit(s_full);
        }
        __syncwarp();
      };
      int requested = 0;
      for (; requested < min(blocks, kStages) && !p.withhold_loads; ++requested) request(requested);
      if (blocks > 0 && wait(q_full, 0)) scores(0);
      for (int i = 0; i < blocks && ok; ++i) {
        const int key0 = kt.tile_index(begin + i) * kBlock;
        const uint32_t v_tile = slot_at(i) + C::kTensor;
        if (key0 + kBlock > kt.hi || (key0 < kt.lo && key0 + kBlock > kt.sink_hi)) {
          // values of keys in nobody's view: zeros
          for (int r = lane; r < kBlock; r += 32) {
            const int key = key0 + r;
            if (!((key < kt.hi && key >= kt.lo) || key < kt.sink_hi)) {
#pragma unroll
              for (int c = 0; c < D / 8; ++c) st_shared_v4(v_tile + r * 128 + c * 16, make_uint4(0, 0, 0, 0));
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (!wait(p_full, i)) break;
        tcgen05_fence_after_sync();
        const uint64_t v_desc = make_smem_desc(v_tile, C::kTensor, 1024);
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < kBlock / 16; ++ks)
            mma_bf16_ts(tmem + C::kColO, tmem + 8 * ks, v_desc + (uint64_t)(ks * ((16 * 128) >> 4)), o_idesc,
                        (i == 0 && ks == 0) ? 0u : 1u);
          mma_commit(o_full);
        }
        __syncwarp();
        // The next scores go over the probabilities: once the product that reads them has completed, the ring slot is free as well.
        if (i + 1 < blocks) {
          if (!wait(o_full, i)) break;
          scores(i + 1);
          if (requested < blocks) request(requested++);
        }
      }
      // Products and copies in flight still use shared and tensor memory: whichever warp gives up, they get a short time to end.
      if (elect_one()) mma_commit(drained);
      __syncwarp();
      volatile int never = 0;
      mbar_wait(drained, 0, &never, nullptr, 0, 20000000ull);
      for (int back = 1; back <= kStages && back <= requested; ++back)
        mbar_wait(full((requested - back) % kStages), ((requested - back) / kStages) & 1u, &never, nullptr, 0, 20000000ull);
    }
  }

  // ------------------------------------------------------------------------ teardown
  __syncwarp();
  tcgen05_fence_before_sync();
  __syncthreads();
  if (warp == kSoftmaxWarps) {
    tcgen05_fence_after_sync();
    tmem_dealloc(tmem, C::kCols);
  }
}

// Launches a kernel of `rows` rows per CTA.
template <typename C, typename... KArgs, typename... Args>
pd_status launch(void (*kernel)(KArgs...), int rows, const pd_paged_attention_desc& d, const Params& p, PerDeviceFlag& smem_allowed,
                 cudaStream_t s, const Args&... args) {
  if (pd_status st = allow_dynamic_smem(kernel, C::kSmem, smem_allowed); st != PD_OK) return st;
  const int64_t tiles = ((int64_t)p.max_q_len * p.group + rows - 1) / rows;
  if (tiles * p.splits > 0x7fffffff) return PD_ERR_BAD_SHAPE;
  launch_pdl(kernel, dim3((unsigned)(tiles * p.splits), d.heads_kv, d.batch), dim3(C::kThreads), C::kSmem, s, args..., p);
  return check_launch();
}

template <int D, pd_dtype T>
pd_status launch_bytes(const pd_paged_attention_desc& d, const Params& p, const Scales& scales, const void* k_cache, const void* v_cache,
                       cudaStream_t s) {
  using Cache = ByteCache<T>;
  using C = WideConfig<D, Cache>;
  const Cache cache{static_cast<const uint8_t*>(k_cache), static_cast<const uint8_t*>(v_cache), d.page_stride, d.slot_stride, d.head_stride, scales};
  static PerDeviceFlag smem_allowed;
  return launch<C>(paged_attention_chunk_kernel<D, Cache>, C::kRows, d, p, smem_allowed, s, cache);
}

}  // namespace

pd_status launch_chunk(const pd_paged_attention_desc& d, const Params& p, const void* k_cache, const void* v_cache, cudaStream_t s) {
  TiledCache cache;
  const int block = d.head_dim == 128 ? kTile : kBlock, box = d.page_size < block ? d.page_size : block;
  if (!make_cache_map(&cache.k, k_cache, d, box) || !make_cache_map(&cache.v, v_cache, d, box)) return PD_ERR_UNSUPPORTED;
  static PerDeviceFlag wide_allowed, narrow_allowed;
  using Wide = WideConfig<128, TiledCache>;
  if (d.head_dim == 128) return launch<Wide>(paged_attention_chunk_kernel<128, TiledCache>, Wide::kRows, d, p, wide_allowed, s, cache);
  return launch<NarrowConfig>(paged_attention_chunk_narrow_kernel, kTile, d, p, narrow_allowed, s, cache.k, cache.v);
}

pd_status launch_chunk_q8(const pd_paged_attention_desc& d, const Params& p, pd_dtype type, const Scales& scales, const void* k_cache,
                          const void* v_cache, cudaStream_t s) {
  if (d.head_dim == 64)
    return type == PD_I8 ? launch_bytes<64, PD_I8>(d, p, scales, k_cache, v_cache, s) : launch_bytes<64, PD_E4M3>(d, p, scales, k_cache, v_cache, s);
  return type == PD_I8 ? launch_bytes<128, PD_I8>(d, p, scales, k_cache, v_cache, s) : launch_bytes<128, PD_E4M3>(d, p, scales, k_cache, v_cache, s);
}

}  // namespace paged
}  // namespace pd
