// Attention over the paged cache for chunks of tokens, on the tcgen05 tensor cores:
//
//   out[t, h] = sum_j softmax_j(scale * q[t, h] . k[j]) v[j],   j visible from token t's position
//
// A CTA takes two consecutive tiles ("slots") of 128 rows of one cache head (a row is a token and one of the query heads
// that share the cache head) and walks the key tiles of 128 keys that any of them sees; both slots read the same K and V
// tiles, which halves what comes from L2.  While one slot's scores are being exponentiated the other slot's products
// run.
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
//                    32 KiB (head_dim 128) stages, K and V in turn.
// Tensor memory: per slot two score buffers of 64 columns and an output of D; with head_dim 128 that is all of it.  Two
// buffers let the scores of the next block be formed while the current ones are exponentiated: the buffer they take was
// last read by the product of the block before.  (With one buffer of 128 columns the softmax warps of a slot waited half
// their time for two products in a row.)
//
// Values of keys in nobody's view may be anything (stale slots of a page, NaN) and would poison the product with
// probability 0 * NaN: in the tiles that hold such keys the issuers overwrite them with zeros first.
// With `splits` > 1 the key tiles are shared out over that many CTAs, whose partial outputs paged_attention_join joins.
#include <type_traits>

#include "paged_cache.cuh"

namespace pd {
namespace paged {
namespace {

constexpr int kTile = 128;             // keys per tile, and rows per slot
constexpr int kBlock = 64;             // keys per score buffer
constexpr int kSoftmaxWarps = 4;       // per slot
constexpr int kStages = 4;
constexpr int kHalf = kTile * 128;     // 64 columns of a tile: 128 lines of 128 bytes
constexpr float kRaise = 8.f;          // powers of two by which a score may exceed the row's reference

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

template <int D>
struct ChunkConfig {
  // head_dim 128: two slots per CTA, one CTA per SM.  head_dim 64: half the tensor memory and a third of the shared memory do
  // for one slot, and two CTAs per SM cover each other's start and end, which weigh more where a window keeps the walk short.
  static constexpr int kSlots = D == 64 ? 1 : 2;
  static constexpr int kCtasPerSm = D == 64 ? 2 : 1;
  static constexpr int kIssuer0 = kSlots * kSoftmaxWarps, kProducer = kIssuer0 + 2 * kSlots;
  static constexpr int kThreads = 32 * (kProducer + 1);
  static constexpr int kRows = kSlots * kTile;
  static constexpr int kTensor = kTile * D * 2;  // a Q, K or V tile
  static constexpr int kSmem = kSlots * kTensor + kStages * kTensor + 1024 /*barriers*/ + 1024 /*alignment*/;
  // tensor-memory columns: score buffer b of slot s at 128 s + 64 b (its probabilities over it, two keys to a column), output
  // of slot s behind them
  static constexpr uint32_t kColO = kSlots * kTile, kCols = kSlots * 256;
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

template <int D>
__global__ void __launch_bounds__(ChunkConfig<D>::kThreads, ChunkConfig<D>::kCtasPerSm)
paged_attention_chunk_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                             const Params p) {
  using C = ChunkConfig<D>;
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
  uint8_t* ctrl = smem_raw + (bars - smem_u32(smem_raw)) + 512;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), kSlots); }
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
      if (view.active) {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(seq.q0 + t) * p.ld_q + (int64_t)head * D);
        const uint32_t dst = sQ + s * C::kTensor + (uint32_t)r * 128u;
#pragma unroll
        for (int c = 0; c < D / 8; ++c)
          st_shared_v4(dst + (c >> 3) * kHalf + (uint32_t)(((c & 7) ^ (r & 7)) << 4), valid ? __ldg(src + c) : make_uint4(0, 0, 0, 0));
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full(s));
      }
      const uint32_t t_lane = tmem + ((uint32_t)(quarter * 32) << 16);
      const uint32_t t_o = t_lane + C::kColO + s * D;
      const uint64_t scale2 = pack_f32x2(p.scale_log2e, p.scale_log2e);
      float m = -INFINITY, l = 0.f;
      uint32_t done = 0;  // blocks of this slot
      bool ok = true;
      for (int b = 0; b < blocks; ++b) {
        const int key0 = block_key(b);
        if (!view.needs(key0)) continue;
        const int buf = done & 1;
        const uint32_t t_s = t_lane + s * kTile + buf * kBlock;
        if (!mbar_wait_warp(s_full(s, buf), (done >> 1) & 1u, abort_flag, p.status, kTimeoutChunkSoftmax)) { ok = false; break; }
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
        const float mx = fmaxf(max3(mx4[0], mx4[1], mx4[2]), mx4[3]) * p.scale_log2e;
        const bool raise = mx > m + kRaise;  // also the first finite score of a row (m = -inf)
        if (__any_sync(0xffffffffu, raise)) {
          const float alpha = raise ? ex2(m - mx) : 1.f;
          if (raise) m = mx;
          l *= alpha;
          if (done > 0) {
            // every product into O so far has to be through with it; the one before last is, or these scores would not be here
            if (!mbar_wait_warp(o_full(s, buf ^ 1), ((done - 1) >> 1) & 1u, abort_flag, p.status, kTimeoutChunkSoftmax)) { ok = false; break; }
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
        const uint64_t nref2 = pack_f32x2(-ref, -ref);
        uint64_t sum2[2] = {0, 0};
        uint32_t pk[32];
        // Groups of sixteen, each group's sums and packing behind the next one's exponentials, in this order: left to the
        // compiler, the special-function unit stood idle between them (894 against 867 us for 4 x 2048 tokens; 790 with no
        // exponentials at all).
        auto scale_group = [&](int g) {
#pragma unroll
          for (int j = 16 * g; j < 16 * g + 16; j += 2) {
            uint32_t(&v)[32] = x[j >> 5];
            float a0, a1;
            unpack_f32x2(fma_f32x2(pack_b32x2(v[j & 31], v[(j & 31) + 1]), scale2, nref2), a0, a1);
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
            sum2[(j >> 1) & 1] = add_f32x2(sum2[(j >> 1) & 1], pack_b32x2(v[j & 31], v[(j & 31) + 1]));
            pk[j / 2] = pack_bf16(__uint_as_float(v[j & 31]), __uint_as_float(v[(j & 31) + 1]));
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
        unpack_f32x2(add_f32x2(sum2[0], sum2[1]), s0, s1);
        l += s0 + s1;
        tmem_st_wait();
        tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(s, buf));
        ++done;
      }
      // ---- the row's output
      if (ok && done > 0) ok = mbar_wait_warp(o_full(s, (done - 1) & 1), ((done - 1) >> 1) & 1u, abort_flag, p.status, kTimeoutChunkSoftmax);
      if (ok && view.active && *abort_flag == 0) {
        tcgen05_fence_after_sync();
        const float inv = l > 0.f ? 1.f / l : 0.f;  // nothing seen: zeros
        const int64_t at = ((int64_t)split * p.tokens + seq.q0 + t) * p.heads_q + head;
        if (p.splits == 1) {
          // through shared memory (this warp's rows of the slot's Q tile, which every product has read), so that a store
          // instruction writes whole rows
          const uint32_t stage = sQ + s * C::kTensor + (uint32_t)(quarter * 32) * 128u;
#pragma unroll
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            if (done > 0) {
              tmem_ld_32x32b_x32(t_o + c, o);
              tmem_ld_wait();
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j)
                w[j] = done > 0 ? pack_bf16(__uint_as_float(o[8 * u + 2 * j]) * inv, __uint_as_float(o[8 * u + 2 * j + 1]) * inv) : 0u;
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
        } else if (done > 0) {
#pragma unroll
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(t_o + c, o);
            tmem_ld_wait();
            if (valid && l > 0.f) {
              float4* dst = reinterpret_cast<float4*>(p.part_o + at * D + c);
#pragma unroll
              for (int u = 0; u < 8; ++u)
                dst[u] = make_float4(__uint_as_float(o[4 * u]) * inv, __uint_as_float(o[4 * u + 1]) * inv,
                                     __uint_as_float(o[4 * u + 2]) * inv, __uint_as_float(o[4 * u + 3]) * inv);
            }
          }
        }
        if (valid && p.splits > 1) p.part_lse[at] = l > 0.f ? m + log2f(l) : -INFINITY;
      }
    } else if (warp == kProducer) {
      // ------------------------------------------------------------------ producer
      const int box = min(p.page_size, kTile);
      const int per_tile = kTile / box, per_batch = 32 / per_tile;
      int page = 0, n = 0;  // n: ring slots requested so far
      bool ok = true;
      for (int i = begin; i < end && ok; ++i) {
        const int in_batch = (i - begin) % per_batch;
        if (in_batch == 0) {
          const int ti = i + lane / per_tile;
          page = ti < end ? page_of(p, b, kt.tile_index(ti) * kTile + (lane % per_tile) * box) : 0;
        }
        const int slot = (kt.tile_index(i) * kTile) & (p.page_size - 1);
        for (int kv = 0; kv < 2; ++kv, ++n) {
          const int stage = n % kStages;
          if (!mbar_wait_warp(empty(stage), ((n / kStages) & 1u) ^ 1u, abort_flag, p.status, kTimeoutChunkProducer)) { ok = false; break; }
          if (elect_one()) mbar_arrive_expect_tx(full(stage), C::kTensor);
          __syncwarp();
          for (int j = 0; j < per_tile; ++j) {
            const int pg = __shfl_sync(0xffffffffu, page, in_batch * per_tile + j);
            if (elect_one()) {
#pragma unroll
              for (int h = 0; h < D / 64; ++h)
                tma_load_4d(ring + stage * C::kTensor + h * kHalf + j * box * 128, kv == 0 ? &tmap_k : &tmap_v, full(stage),
                            h * 64, slot, kvh, pg);
            }
            __syncwarp();
          }
        }
      }
      if (!ok) {
        // leave no copy in flight: give the last request of every stage a short time to land
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
        ok = ok && mbar_wait_warp(bar, parity & 1u, abort_flag, p.status, kTimeoutChunkMma);
        return ok;
      };
      constexpr uint64_t kBlockStep = (kBlock * 128) >> 4;  // descriptor step from a tile's first block to its second
      if (((warp - kIssuer0) & 1) == 0) {
        // ---- scores; K tile t is in ring slot 2 t
        constexpr uint32_t idesc = make_idesc_bf16(kTile, kBlock, false, false);
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
        constexpr uint32_t idesc = make_idesc_bf16(kTile, D, false, true);  // V is MN-major
        for (int b = 0; b < blocks && ok; ++b) {
          const int n = b | 1, stage = n % kStages;
          const int key0 = block_key(b);
          if ((b & 1) == 0) {
            if (!wait(full(stage), n / kStages)) break;
            if ((view.needs(key0) || view.needs(key0 + kBlock)) &&
                (key0 + kTile > kt.hi || (key0 < kt.lo && key0 + kTile > kt.sink_hi))) {
              // values of keys in nobody's view: zeros (both slots' issuers write the same; neither's product reads the
              // tile before its own are in)
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
      if (!ok) {
        // products in flight still read shared and tensor memory: give them a short time to end
        if (elect_one()) mma_commit(drained(warp - kIssuer0));
        __syncwarp();
        volatile int never = 0;
        mbar_wait(drained(warp - kIssuer0), 0, &never, nullptr, 0, 20000000ull);
      }
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

template <int D>
pd_status launch(const pd_paged_attention_desc& d, const Params& p, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t s) {
  using C = ChunkConfig<D>;
  static PerDeviceFlag smem_allowed;
  if (pd_status st = allow_dynamic_smem(paged_attention_chunk_kernel<D>, C::kSmem, smem_allowed); st != PD_OK) return st;
  const int64_t tiles = ((int64_t)p.max_q_len * p.group + C::kRows - 1) / C::kRows;
  if (tiles * p.splits > 0x7fffffff) return PD_ERR_BAD_SHAPE;
  launch_pdl(paged_attention_chunk_kernel<D>, dim3((unsigned)(tiles * p.splits), d.heads_kv, d.batch), dim3(C::kThreads),
             C::kSmem, s, tk, tv, p);
  return check_launch();
}

}  // namespace

pd_status launch_chunk(const pd_paged_attention_desc& d, const Params& p, const void* k_cache, const void* v_cache, cudaStream_t s) {
  CUtensorMap tk, tv;
  const int box = d.page_size < kTile ? d.page_size : kTile;
  if (!make_cache_map(&tk, k_cache, d, box) || !make_cache_map(&tv, v_cache, d, box)) return PD_ERR_UNSUPPORTED;
  return d.head_dim == 64 ? launch<64>(d, p, tk, tv, s) : launch<128>(d, p, tk, tv, s);
}

}  // namespace paged
}  // namespace pd
