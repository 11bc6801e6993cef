// Attention over an 8-bit paged cache for few rows per cache head (single tokens, drafts, short chunks):
//
//   out[t, h] = sum_j softmax_j(scale * ks_j * (q[t, h] . k8[j])) vs_j v8[j],   j visible from token t's position
//
// Bound: HBM, at half the bytes per key of a bf16 cache, so that twice the keys have to go through the SM in the same time.  How
// tiles are dealt out to CTAs, and joined, is that of the bf16 kernel (paged_rows.cuh); what differs is everything in between.
//
// Arithmetic: the stored bytes become fp16, exactly, in a few instructions per word, and go through mma.sync as the A operand:
// S^T = K Q^T and O^T = V^T P^T, keys (or elements of a head) along the 16 rows of the instruction and query rows along its 8
// columns.  A tile of up to 8 rows, the usual single token, then costs half of what it does with the rows along the 16.  A byte
// is converted once per warp, however many rows the warp has; words are taken as ldmatrix delivers them, bytes 0 and 2 as one
// operand register and 1 and 3 as the other, which permutes the elements of a head alike in K and Q, and in O.
//   Q: multiplied by a power of two that takes the largest magnitude of a warp's rows to [2^14, 2^15), which is exact in fp16 down to 2^-28
//      of it (and off by 2^-40 of it below); the power is taken back in the scale of the scores.  Rows that are more than 2^12 apart
//      have a power each, so that a row's queries are off by 2^-28 of its own largest at most, whatever the others hold.
//   S: fp32, times ks_j.
//   P: exponentials, fp32, times vs_j and a power of two that keeps them below 2^15, rounded to fp16 (2^-11 of each; what is
//      2^-24 and less of the largest is off by up to 2^-35 of that).  The power follows the largest vs_j that the row has seen.
//   O: fp32 sums.  The row sums of the exponentials are fp32, too, and of the unrounded ones.
//
// A producer warp copies key tiles by TMA, one box per page and tensor, and their scales with one 4-byte copy per block; K (with
// all scales) and V of a tile are a stage of the ring each.  Four consumer warps take 32 keys of a tile each.  In the usual layout a
// slot's heads lie beside each other, 64 or 128 bytes each, and a tile of one head would take that much of every slot: DRAM
// delivered 4.2 TB/s so.  So the warps take up to four neighbouring heads, and a box has the rows of all of them; where there are fewer
// heads, warps share the keys of a tile, and more than 16 rows are shared by two or four warps.  A warp keeps a reference maximum of its
// own, raised when a score exceeds it by 2^4; warps with the same rows meet at the end of a piece.
//   64 single tokens over 200 to 8192 keys, 32/8 heads of 128, int8: 104 us, 81 % of the copy rate (bf16 cache: 186); the loads alone
//   97 to 99.  16 x 5 tokens over up to 8192 keys, e4m3: 69 us, where the loads alone take 38.  No unit is full there (issue slots 42 %,
//   tensor cores 32 %, DRAM 29 %): eight warps to an SM do not hide a warp's chain of conversions, products and softmax.
#pragma once

#include <type_traits>

#include "cache_q8.cuh"
#include "paged_rows.cuh"

namespace pd {
namespace paged {
namespace {

constexpr int kKeys = 32;        // of a tile, per warp
constexpr int kConsumers = 4;    // warps
constexpr int kThreads = 32 * (kConsumers + 1);
constexpr float kRaise = 4.f;    // powers of two by which a score may exceed the reference
constexpr float kLift = 90.f;    // 2^(kRaise + kLift) times the keys that there can be is in fp32's range
constexpr float kTopP = 2048.f;  // 2^(15 - kRaise): the largest vs_j times the power of two that goes with P

// H cache heads side by side, WK warps that share a tile's keys, WR that share the rows; NR groups of 8 rows to a warp.
template <int D, int NR, int H, int WK, int WR>
struct Q8Config {
  static_assert(H * WK * WR == kConsumers);
  static constexpr int kTile = kKeys * WK;              // keys
  static constexpr int kGroupRows = 8 * NR;             // rows of a warp
  static constexpr int kRows = kGroupRows * WR;
  static constexpr int kStageBytes = H * kTile * D;     // K or V of a tile
  static constexpr int kScaleBytes = 2 * H * kTile * 4; // a scale per key at most, for K and for V
  // From 24 rows on the queries' fragments stay in shared memory, and a warp takes its 32 keys 16 at a time: 168 registers a thread
  // hold the accumulators of 24 rows and little else.
  static constexpr bool kLean = NR > 2;
  static constexpr int kQ = kLean ? kConsumers * NR * (D / 16) * 256 : 0;
  static constexpr int kExchange = WK > 1 ? H * WR * (WK / 2) * 512 * (D / 16 + 1) : 0;  // half the warps' results for 8 rows
  static constexpr int kRowBytes = 2 * kGroupRows * 4;  // two floats for each of a warp's rows
  static constexpr int kControl = 256 /*barriers*/ + kConsumers * kRowBytes;
  static constexpr int kPerCta = 113 * 1024 - kControl - 1024 /*alignment*/;             // two CTAs per SM
  static constexpr int kFit = (kPerCta - kExchange - kQ) / (kStageBytes + kScaleBytes);
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr int kSmem = kStages * (kStageBytes + kScaleBytes) + kExchange + kQ + kControl + 1024;
  static_assert(2 * (kSmem + 1024) <= 228 * 1024 && kStages >= 4);
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void copy_async_4(uint32_t dst, const float* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
// An arrival on `bar` (counted in its initialisation) once this thread's copies so far have landed.
__device__ __forceinline__ void arrive_after_copies(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// The power of two above v, within what fp32 has as a power of two times kTopP; 0 for 0.
__device__ __forceinline__ float power_above(float v) {
  return v > 0.f ? __uint_as_float(min(max((__float_as_uint(v) >> 23) + 1u, 27u), 254u) << 23) : 0.f;
}
// How many powers of two `own` is below `top`, as far as a sum of exponentials can be raised by; all of them for 0.
__device__ __forceinline__ float lift(float top, float own) {
  return own > 0.f ? fminf((float)((int)(__float_as_uint(top) >> 23) - (int)(__float_as_uint(own) >> 23)), kLift) : kLift;
}

template <pd_dtype T, int D, int NR, int H, int WK, int WR>
__global__ void __launch_bounds__(kThreads, 2)
paged_attention_q8_rows_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const Params p,
                               const Scales scales) {
  using C = Q8Config<D, NR, H, WK, WR>;
  constexpr int kTile = C::kTile, kTileShift = kTile == 32 ? 5 : kTile == 64 ? 6 : 7;
  constexpr bool kAdjacent = T != PD_I8;  // K's words: bytes 0 and 1 together, else 0 and 2
  extern __shared__ uint8_t smem_raw[];
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t scale_ring = ring + C::kStages * C::kStageBytes, exchange_at = scale_ring + C::kStages * C::kScaleBytes;
  float* exchange = reinterpret_cast<float*>(smem_raw + (exchange_at - smem_u32(smem_raw)));
  const uint32_t sq = exchange_at + C::kExchange + (threadIdx.x >> 5) * (C::kQ / kConsumers) + (threadIdx.x & 31) * 8;  // this lane's queries
  const uint32_t bars = exchange_at + C::kExchange + C::kQ;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 64u + 8u * s; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + (bars - smem_u32(smem_raw)) + 128);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto row_power = [&](int r) { return bars + 256u + (uint32_t)(warp * C::kRowBytes + 4 * r); };  // of a consumer warp's row: what its scores still need
  auto row_top = [&](int r) { return row_power(C::kGroupRows + r); };  // a power of two, at least the largest vs_j that it has seen

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(full(s), 1 + 32); mbar_init(empty(s), kConsumers); }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == kConsumers && lane == 0) { prefetch_tensormap(&tmap_k); prefetch_tensormap(&tmap_v); }
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();

  Piece w;  // (w.kvh counts groups of H cache heads)
  int start, stop, share;
  if (!first_piece<kThreads, kTile>(p, blockIdx.x, w, start, stop, share)) return;
  const int box_shift = min(p.page_shift, kTileShift);      // slots of a page's box
  const int scale_shift = min(scales.shift, kTileShift), blocks = kTile >> scale_shift;  // scales of a tile and head

  if (warp == kConsumers) {
    // ------------------------------------------------------------------ producer
    // Per stage: kTile / page_size pages (or a part of one), each a box of slots of H heads that a lane of its own requests.  The
    // lanes hold the pages of `per_batch` tiles, and the table's entries for as many behind them.
    const int tile_shift = kTileShift - box_shift, batch_shift = 5 - tile_shift;
    const int in_tile = lane & ((1 << tile_shift) - 1);
    bool ok = !p.withhold_loads;
    int stage = 0, n = 0;  // stages requested so far
    uint32_t phase = 1;
    auto request = [&](const CUtensorMap* map, int slot, int pg) {  // waits for the stage, and asks for one of the tensors
      if (!mbar_wait_warp(empty(stage), phase, abort_flag, p.status, kTimeoutRowsProducer, p.wait_limit_ns)) return false;
      if (lane == 0) mbar_arrive_expect_tx(full(stage), C::kStageBytes);
      __syncwarp();
      if (lane < (1 << tile_shift))
        tma_load_4d(ring + stage * C::kStageBytes + (uint32_t)(lane << box_shift) * (H * D), map, full(stage), 0, slot, w.kvh * H, pg);
      return true;
    };
    auto advance = [&]() {
      arrive_after_copies(full(stage));
      ++n;
      if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
    };
    while (ok) {
      const int end = min(w.end, w.tiles.n);
      auto entry_of = [&](int i) {  // of the lane's tile and page in the batch that begins with tile i; -1: none
        const int ti = i + (lane >> tile_shift);
        const int at = ti < end ? (w.tiles.tile_index(ti) * kTile + (in_tile << box_shift)) >> p.page_shift : p.max_pages;
        int e = -1;
        if (at < p.max_pages) e = __ldg(p.block_table + (int64_t)w.b * p.max_pages + at);
        return e;
      };
      int ahead = entry_of(w.begin), page = 0;
      for (int i = w.begin; i < end; ++i) {
        const int in_batch = (i - w.begin) & ((1 << batch_shift) - 1);
        if (in_batch == 0) {
          page = (unsigned)ahead < (unsigned)p.num_pages ? ahead : p.num_pages;
          ahead = entry_of(i + (1 << batch_shift));
        }
        const int slot = (w.tiles.tile_index(i) * kTile) & (p.page_size - 1);  // 0 unless a page holds several tiles
        const int pg = __shfl_sync(0xffffffffu, page, (in_batch << tile_shift) + in_tile);
        if (!request(&tmap_k, slot, pg)) { ok = false; break; }
        for (int e0 = 0; e0 < H * blocks; e0 += 32) {
          const int e = e0 + lane, h = e / blocks, key = (e - h * blocks) << scale_shift;  // (a power of two)
          const int mine = __shfl_sync(0xffffffffu, page, (in_batch << tile_shift) + (key >> box_shift));
          if (e < H * blocks) {
            const bool there = mine < p.num_pages;
            const int64_t at = there ? scales.at(mine, w.kvh * H + h, slot + (key & ((1 << box_shift) - 1))) : 0;
            const uint32_t dst = scale_ring + stage * C::kScaleBytes + 4u * e;
            copy_async_4(dst, scales.k + at, there);
            copy_async_4(dst + 4u * H * kTile, scales.v + at, there);
          }
        }
        advance();
        if (!request(&tmap_v, slot, pg)) { ok = false; break; }
        advance();
      }
      if (!ok || !next_piece<kTile>(p, w, stop)) break;
    }
    // Leave no copy in flight, whichever warp gives up: the last request of every stage gets a short time to land.
    volatile int never = 0;
    for (int back = 1; back <= C::kStages && back <= n; ++back)
      mbar_wait(full((n - back) % C::kStages), ((n - back) / C::kStages) & 1u, &never, nullptr, 0, 20000000ull);
    return;
  }

  // ------------------------------------------------------------------- consumers
  const int hs = warp % H, wk = warp / H % WK, wr = warp / (H * WK);
  constexpr int KS = D / 16, MT = D / 16;  // steps of 16 elements; tiles of 16 elements
  constexpr int HB = C::kLean ? 1 : 2;     // tiles of 16 keys at a time
  const int g = lane >> 2, i4 = lane & 3;
  // this lane's ldmatrix rows (a key of either 16 of the warp's) within a stage, and which of two neighbouring 16-byte chunks
  const int mat_chunk = lane >> 4;
  uint32_t mat_row[2];
  int mat_swizzle[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int key = wk * kKeys + 16 * h + (lane & 15);
    mat_row[h] = (uint32_t)(((((key >> box_shift) * H + hs) << box_shift) + (key & ((1 << box_shift) - 1))) * D);
    mat_swizzle[h] = D == 128 ? key & 7 : (key >> 1) & 3;
  }
  auto chunk_at = [&](uint32_t tensor, int h, int chunk) { return tensor + mat_row[h] + (uint32_t)((chunk ^ mat_swizzle[h]) << 4); };
  int stage = 0;
  uint32_t phase = 0;
  auto advance = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(empty(stage));
    if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
  };
  for (int piece = 0;; ++piece) {
    const int first_pos = w.seq.pos0, last_pos = w.seq.pos0 + w.seq.n - 1;
    const int kvh = w.kvh * H + hs;
    const KeyTiles& kt = w.tiles;
    // ---- queries: row 8 r + g of the warp's, elements 16 k + 4 i ... + 3 of it
    uint32_t qf[C::kLean ? 1 : NR][KS][2];
    float score_scale;
    bool apart;
    {
      auto source = [&](int r) {
        const int row = min(wr * C::kGroupRows + 8 * r + g, w.rows - 1);  // (rows beyond the last repeat it and are not stored)
        const int t = row / p.group;
        return p.q + (int64_t)(w.seq.q0 + t) * p.ld_q + (int64_t)(kvh * p.group + row % p.group) * D + 4 * i4;
      };
      auto load = [&](const __nv_bfloat16* src, int k) { return *reinterpret_cast<const uint2*>(src + 16 * k); };
      // The largest exponent e of the rows goes to 14: times 2^(14 - e), within what fp32 has as a power of two and its reciprocal.  Rows
      // more than 2^kNear apart (one that is infinite or not a number, too) each get a power of their own: the middle one of the
      // reciprocals goes with the scale of the scores, the rest is taken back in each row's scores.
      constexpr int kNear = 12, kNone = 127;  // (rows of zeros take whatever the others have)
      uint32_t most[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) {  // (all loads before the first exchange)
        const __nv_bfloat16* src = source(r);
        most[r] = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint2 v = load(src, k);
          most[r] = max(most[r], max(max(v.x & 0x7fff0000u, v.x << 16 & 0x7fff0000u), max(v.y & 0x7fff0000u, v.y << 16 & 0x7fff0000u)));
        }
      }
      int shift[NR], least = kNone, largest = -126;
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        most[r] = max(most[r], __shfl_xor_sync(0xffffffffu, most[r], 1));
        most[r] = max(most[r], __shfl_xor_sync(0xffffffffu, most[r], 2));
        shift[r] = most[r] == 0 ? kNone : min(max(14 + 127 - (int)(most[r] >> 23), -126), 126);
        least = min(least, shift[r]);
        if (most[r] != 0) largest = max(largest, shift[r]);
      }
      least = __reduce_min_sync(0xffffffffu, least);
      largest = __reduce_max_sync(0xffffffffu, largest);
      apart = largest - least > kNear;
      const int middle = least == kNone ? 0 : apart ? (least + largest) >> 1 : least;
#pragma unroll
      for (int r = 0; r < NR; ++r)
        if (!apart || shift[r] == kNone) shift[r] = middle;
      score_scale = p.scale_log2e * __uint_as_float((uint32_t)(127 - middle) << 23);
      __syncwarp();
#pragma unroll
      for (int r = 0; r < NR; ++r)
        if (i4 == 0) st_shared_f32(row_power(8 * r + g), __uint_as_float((uint32_t)(127 + middle - shift[r]) << 23));
      __syncwarp();
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const __nv_bfloat16* src = source(r);
        const float up = __uint_as_float((uint32_t)(127 + shift[r]) << 23);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint2 v = load(src, k);
          const float x0 = __uint_as_float(v.x << 16) * up, x1 = __uint_as_float(v.x & 0xffff0000u) * up;
          const float x2 = __uint_as_float(v.y << 16) * up, x3 = __uint_as_float(v.y & 0xffff0000u) * up;
          const uint32_t b0 = kAdjacent ? pack_half(x0, x1) : pack_half(x0, x2), b1 = kAdjacent ? pack_half(x2, x3) : pack_half(x1, x3);
          if constexpr (C::kLean) {
            asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(sq + (uint32_t)((r * KS + k) * 256)), "r"(b0), "r"(b1) : "memory");
          } else {
            qf[r][k][0] = b0;
            qf[r][k][1] = b1;
          }
        }
      }
    }
    // positions of the rows 8 r + 2 i and + 1, which this lane has scores of
    int pos[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) pos[r][e] = w.seq.pos0 + min(wr * C::kGroupRows + 8 * r + 2 * i4 + e, w.rows - 1) / p.group;
    float o[MT][NR][4];
#pragma unroll
    for (int d = 0; d < MT; ++d)
#pragma unroll
      for (int r = 0; r < NR; ++r) o[d][r][0] = o[d][r][1] = o[d][r][2] = o[d][r][3] = 0.f;
    float m[NR][2], l[NR][2];  // references (in powers of two), this lane's part of the sums
#pragma unroll
    for (int r = 0; r < NR; ++r) { m[r][0] = m[r][1] = -INFINITY; l[r][0] = l[r][1] = 0.f; }
    // O is in units of 1 / v_unit: kTopP over a power of two that is at least the largest vs_j that a row has seen so far (0: none).  Rows
    // differ in what they see, so each has such a power of its own (row_top, in shared memory; their smallest: least_top), and its reference
    // lies below its largest score by what its own is below the warp's: the products then fill fp16's range for every row.
    float v_unit = 0.f, least_top = 0.f;

    bool failed = false;
    const int end = min(w.end, kt.n);
    // Compiled twice, so that rows that are not apart, as they hardly ever are, have no instruction for it: in one, 64 x 4096 keys took
    // 141 us against 135 with 16 rows of 128, 240 against 232 with 32.  Up to 8 rows have the registers for it, and the longer way to the
    // code costs a first call 2 us.
    constexpr bool kTwice = NR > 1;
    // Rows of one power are raised in a path of their own, which is most of what short walks see of it (16 x 2048 keys, 20 rows of 64: 30 against
    // 32 us); the form of 24 rows of 128, for long walks alone, has no registers to spare (64 x 4096: 203 against 196).
    constexpr bool kLevel = !(C::kLean && D == 128);
    auto walk = [&](auto own_powers) {
      for (int i = w.begin; i < end; ++i) {
        // (a warp that gives up goes on to the barrier below, if there is one, which tells the others)
        if (!mbar_wait_warp(full(stage), phase, abort_flag, p.status, kTimeoutRowsConsumer, p.wait_limit_ns)) { failed = true; break; }
        const uint32_t sk = ring + stage * C::kStageBytes, sc = scale_ring + stage * C::kScaleBytes + 4u * (uint32_t)(hs * blocks);
        const int key0 = kt.tile_index(i) * kTile + wk * kKeys;
        uint32_t sv = 0;
        if constexpr (HB == 1) {  // both at once, and both are given back at the end
          const bool wraps = stage + 1 == C::kStages;
          sv = ring + (wraps ? 0 : stage + 1) * C::kStageBytes;
          if (!mbar_wait_warp(full(wraps ? 0 : stage + 1), wraps ? phase ^ 1u : phase, abort_flag, p.status, kTimeoutRowsConsumer, p.wait_limit_ns)) { failed = true; break; }
        }
        // keys outside a row's view; whole tiles in everybody's view skip this
        const int last_key = key0 + kKeys - 1;
        const bool whole = last_key <= first_pos && last_key < w.seq.length && (p.window == 0 || key0 > last_pos - p.window || last_key < p.sinks);
        auto in_view = [&](int key) { return (key < kt.hi && key >= kt.lo) || key < kt.sink_hi; };  // of some row
#pragma unroll 1
        for (int h0 = 0; h0 < 2; h0 += HB) {
          // ---- S^T = K Q^T, one or two tiles of 16 keys
          float s[HB][NR][4];
#pragma unroll
          for (int h = 0; h < HB; ++h) {
#pragma unroll
            for (int r = 0; r < NR; ++r) s[h][r][0] = s[h][r][1] = s[h][r][2] = s[h][r][3] = 0.f;
            // words of keys 0-7 and 8-15, of two steps' 16 elements each; lean: these and the queries are asked for a step ahead
            uint32_t kw[2][4], qb[2][NR][2];
            auto keys_of = [&](int k) { ldmatrix_x4(chunk_at(sk, h0 + h, k + mat_chunk), kw[(k >> 1) & 1]); };
            auto queries_of = [&](int k) {
#pragma unroll
              for (int r = 0; r < NR; ++r)
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(qb[k & 1][r][0]), "=r"(qb[k & 1][r][1]) : "r"(sq + (uint32_t)((r * KS + k) * 256)));
            };
            if constexpr (C::kLean) {
              keys_of(0);
              queries_of(0);
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              if constexpr (C::kLean) {
                if (k % 2 == 0 && k + 2 < KS) keys_of(k + 2);
                if (k + 1 < KS) queries_of(k + 1);
              } else if (k % 2 == 0) {
                keys_of(k);
              }
              const uint32_t* words = kw[(k >> 1) & 1] + 2 * (k & 1);
              uint32_t a0, a1, a2, a3;
              q8_word_to_half<T, kAdjacent>(words[0], a0, a2);
              q8_word_to_half<T, kAdjacent>(words[1], a1, a3);
#pragma unroll
              for (int r = 0; r < NR; ++r) {
                if constexpr (C::kLean) mma_f16(s[h][r], a0, a1, a2, a3, qb[k & 1][r][0], qb[k & 1][r][1]);
                else mma_f16(s[h][r], a0, a1, a2, a3, qf[r][k][0], qf[r][k][1]);
              }
            }
          }
          // ---- scales of this lane's keys 16 h + 8 e + g
          float ks[HB][2], vs[HB][2];
#pragma unroll
          for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t at = sc + 4u * (uint32_t)((wk * kKeys + 16 * (h0 + h) + 8 * e + g) >> scale_shift);
              ks[h][e] = ld_shared_f32(at) * score_scale;
              vs[h][e] = ld_shared_f32(at + 4u * H * kTile);
            }
          if constexpr (HB == 2) advance();
#pragma unroll
          for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[h][r][e] *= ks[h][e >> 1];
          if (!whole) {
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = key0 + 16 * (h0 + h) + 8 * (e >> 1) + g;
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                  const int at = pos[r][e & 1];
                  const bool seen = key <= at && key < w.seq.length && (p.window == 0 || key > at - p.window || key < p.sinks);
                  if (!seen) s[h][r][e] = -INFINITY;
                }
                if (!in_view(key)) vs[h][e >> 1] = 0.f;
              }
          }
          if (kTwice ? own_powers.value : apart) {
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float power = ld_shared_f32(row_power(8 * r + 2 * i4 + e));
#pragma unroll
                for (int h = 0; h < HB; ++h) {
                  s[h][r][e] *= power;
                  s[h][r][e + 2] *= power;
                }
              }
          }
          // ---- references
          float v_most = fmaxf(vs[0][0], vs[0][1]);
          if constexpr (HB == 2) v_most = fmaxf(v_most, fmaxf(vs[1][0], vs[1][1]));
          float mx[NR][2];
          bool raise = v_most > least_top;
#pragma unroll
          for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              mx[r][e] = fmaxf(s[0][r][e], s[0][r][e + 2]);
              if constexpr (HB == 2) mx[r][e] = fmaxf(mx[r][e], fmaxf(s[1][r][e], s[1][r][e + 2]));
              raise |= mx[r][e] > m[r][e] + kRaise;  // also the first finite score of a row (m = -inf)
            }
          if (__any_sync(0xffffffffu, raise)) {
            const float most = warp_max(v_most), top0 = v_unit > 0.f ? kTopP / v_unit : 0.f, top1 = fmaxf(top0, power_above(most));
            const float down = top1 > 0.f ? top0 / top1 : 1.f;
            const bool level = __all_sync(0xffffffffu, least_top == top0);  // all rows' powers are the warp's
            v_unit = top1 > 0.f ? kTopP / top1 : 0.f;
            if (kLevel && __builtin_expect(level && (top1 == top0 || whole || first_pos == last_pos), 1)) {  // and stay so: all see what there is to see here
              least_top = top1;
#pragma unroll
              for (int r = 0; r < NR; ++r) {
                float alpha[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  float top = mx[r][e];
#pragma unroll
                  for (int x = 4; x < 32; x *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                  const bool up = top > m[r][e] + kRaise;
                  alpha[e] = up ? ex2(m[r][e] - top) : 1.f;
                  if (up) m[r][e] = top;
                  l[r][e] *= alpha[e];
                  alpha[e] *= down;
                }
#pragma unroll
                for (int d = 0; d < MT; ++d) {
                  o[d][r][0] *= alpha[0]; o[d][r][1] *= alpha[1]; o[d][r][2] *= alpha[0]; o[d][r][3] *= alpha[1];
                }
              }
            } else {
              least_top = INFINITY;
              __syncwarp();  // (what was written here the last time is there)
#pragma unroll
              for (int r = 0; r < NR; ++r) {
                float alpha[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  float top = mx[r][e], seen = 0.f;
#pragma unroll
                  for (int h = 0; h < HB; ++h)
#pragma unroll
                    for (int x = 0; x < 2; ++x) seen = s[h][r][e + 2 * x] > -INFINITY ? fmaxf(seen, vs[h][x]) : seen;
#pragma unroll
                  for (int x = 4; x < 32; x *= 2) {
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                    seen = fmaxf(seen, __shfl_xor_sync(0xffffffffu, seen, x));
                  }
                  const uint32_t at = row_top(8 * r + 2 * i4 + e);
                  const float own0 = level ? top0 : ld_shared_f32(at), own1 = fmaxf(own0, power_above(seen));
                  const float lift0 = level ? 0.f : lift(top0, own0), lift1 = lift(top1, own1), peak = m[r][e] + lift0;
                  float ref = lift1 == lift0 ? m[r][e] : peak - lift1;
                  if (top > peak + kRaise) ref = top - lift1;
                  alpha[e] = ref == m[r][e] ? 1.f : ex2(m[r][e] - ref);
                  m[r][e] = ref;
                  l[r][e] *= alpha[e];
                  alpha[e] *= down;
                  least_top = fminf(least_top, own1);
                  __syncwarp();
                  if (g == 0) st_shared_f32(at, own1);
                }
#pragma unroll
                for (int d = 0; d < MT; ++d) {
                  o[d][r][0] *= alpha[0]; o[d][r][1] *= alpha[1]; o[d][r][2] *= alpha[0]; o[d][r][3] *= alpha[1];
                }
              }
            }
          }
          // ---- P^T: exponentials, and times vs_j in fp16
          uint32_t pf[HB][NR][2];
#pragma unroll
          for (int h = 0; h < HB; ++h) {
            const float v0 = vs[h][0] * v_unit, v1 = vs[h][1] * v_unit;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              // a row that has seen nothing yet is referred to 0: its exponentials are 2^-inf = 0
              const float r0 = m[r][0] == -INFINITY ? 0.f : m[r][0], r1 = m[r][1] == -INFINITY ? 0.f : m[r][1];
              const float e0 = ex2(s[h][r][0] - r0), e1 = ex2(s[h][r][1] - r1), e2 = ex2(s[h][r][2] - r0), e3 = ex2(s[h][r][3] - r1);
              l[r][0] += e0 + e2;
              l[r][1] += e1 + e3;
              pf[h][r][0] = transpose_8x8(pack_half(e0 * v0, e1 * v0));
              pf[h][r][1] = transpose_8x8(pack_half(e2 * v1, e3 * v1));
            }
          }
          // ---- O^T += V^T P^T
          if constexpr (HB == 2) {
            if (!mbar_wait_warp(full(stage), phase, abort_flag, p.status, kTimeoutRowsConsumer, p.wait_limit_ns)) { failed = true; break; }
            sv = ring + stage * C::kStageBytes;
          }
#pragma unroll
          for (int h = 0; h < HB; ++h) {
            // Values of keys in nobody's view may be any bits, NaN among them: zeroed, since 0 * NaN is NaN.  A word holds two
            // elements of key 2 i (of eight) and two of key 2 i + 1.
            uint32_t mask0 = 0xffffffffu, mask1 = 0xffffffffu;
            if (!whole) {
              auto half = [&](int key) { return in_view(key) ? 0xffffu : 0u; };
              const int key = key0 + 16 * (h0 + h) + 2 * i4;
              mask0 = half(key) | half(key + 1) << 16;
              mask1 = half(key + 8) | half(key + 9) << 16;
            }
            uint32_t vw[2][4];  // words of keys 0-7 and 8-15, of 16 elements and the next ones
            auto values_of = [&](int d) { ldmatrix_x4_trans(chunk_at(sv, h0 + h, d + mat_chunk), vw[(d >> 1) & 1]); };
            values_of(0);
#pragma unroll
            for (int d = 0; d < MT; d += 2) {
              if (d + 2 < MT) values_of(d + 2);
              uint32_t(&words)[4] = vw[(d >> 1) & 1];
              if (!whole) { words[0] &= mask0; words[1] &= mask1; words[2] &= mask0; words[3] &= mask1; }
#pragma unroll
              for (int d2 = 0; d2 < 2; ++d2) {
                uint32_t a0, a1, a2, a3;
                q8_word_to_half<T, false>(words[2 * d2], a0, a1);
                q8_word_to_half<T, false>(words[2 * d2 + 1], a2, a3);
#pragma unroll
                for (int r = 0; r < NR; ++r) mma_f16(o[d + d2][r], a0, a1, a2, a3, pf[h][r][0], pf[h][r][1]);
              }
            }
          }
        }
        if (failed) break;
        if constexpr (HB == 1) advance();
        advance();
      }
    };
    if (!kTwice || __builtin_expect(!apart, 1)) walk(std::false_type{});
    else walk(std::true_type{});
    float unit = v_unit > 0.f ? 1.f / v_unit : 0.f;
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int x = 4; x < 32; x *= 2) l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], x);
    if constexpr (WK == 1) {
      if (failed) break;
    } else {
      // (the last piece's exchange has been read by then)
      if (barrier_any<32 * kConsumers>(failed)) break;
      // The warps with the same rows: the upper half's results go, lane by lane and 8 rows at a time, into the lower half's registers,
      // until one is left.
#pragma unroll
      for (int half = WK / 2; half > 0; half /= 2) {
        const int step = H * WR * half * 32 * 4;  // floats
        float* mine = exchange + (((wr * H + hs) * half + wk % half) * 32 + lane) * 4;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          if (wk >= half && wk < 2 * half) {
#pragma unroll
            for (int d = 0; d < MT; ++d)
              *reinterpret_cast<float4*>(mine + d * step) = make_float4(o[d][r][0] * unit, o[d][r][1] * unit, o[d][r][2] * unit, o[d][r][3] * unit);
            *reinterpret_cast<float4*>(mine + MT * step) = make_float4(m[r][0], m[r][1], l[r][0], l[r][1]);
          }
          asm volatile("bar.sync 1, %0;" ::"n"(32 * kConsumers) : "memory");
          if (wk < half) {
            const float4 other = *reinterpret_cast<const float4*>(mine + MT * step);
            const float om[2] = {other.x, other.y}, ol[2] = {other.z, other.w};
            float a[2], b[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float top = fmaxf(m[r][e], om[e]);
              a[e] = m[r][e] == -INFINITY ? 0.f : ex2(m[r][e] - top);
              b[e] = om[e] == -INFINITY ? 0.f : ex2(om[e] - top);
              m[r][e] = top;
              l[r][e] = l[r][e] * a[e] + ol[e] * b[e];
              a[e] *= unit;
            }
#pragma unroll
            for (int d = 0; d < MT; ++d) {
              const float4 v = *reinterpret_cast<const float4*>(mine + d * step);
              o[d][r][0] = o[d][r][0] * a[0] + v.x * b[0];
              o[d][r][1] = o[d][r][1] * a[1] + v.y * b[1];
              o[d][r][2] = o[d][r][2] * a[0] + v.z * b[0];
              o[d][r][3] = o[d][r][3] * a[1] + v.w * b[1];
            }
          }
          asm volatile("bar.sync 1, %0;" ::"n"(32 * kConsumers) : "memory");
        }
        unit = 1.f;
      }
    }
    // ---- the rows 8 r + 2 i and + 1, elements 16 d + 2 g and + 1: to the output, or to the workspace
    const bool complete = w.begin == 0 && w.end == w.weight;
    const int part = 2 * blockIdx.x + (piece > 0 ? 1 : 0);  // a piece that is neither the CTA's first nor its last is complete
    if (wk == 0) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = wr * C::kGroupRows + 8 * r + 2 * i4 + e;
          const float inv = l[r][e] > 0.f ? unit / l[r][e] : 0.f;  // nothing seen: zeros
          if (row < w.rows) {
            if (complete) {
              const int t = row / p.group;
              __nv_bfloat16* to = p.out + (int64_t)(w.seq.q0 + t) * p.ld_out + (int64_t)(kvh * p.group + row - t * p.group) * D + 2 * g;
#pragma unroll
              for (int d = 0; d < MT; ++d) *reinterpret_cast<uint32_t*>(to + 16 * d) = pack_bf16(o[d][r][e] * inv, o[d][r][2 + e] * inv);
            } else {
              const int64_t at = ((int64_t)part * H + hs) * C::kRows + row;
              if (l[r][e] > 0.f) {
#pragma unroll
                for (int d = 0; d < MT; ++d) *reinterpret_cast<float2*>(p.part_o + at * D + 16 * d + 2 * g) = make_float2(o[d][r][e] * inv, o[d][r][2 + e] * inv);
              }
              if (g == 0) p.part_lse[at] = l[r][e] > 0.f ? m[r][e] + log2f(l[r][e]) : -INFINITY;
            }
          }
        }
      if (wr == 0 && lane == 0 && w.begin == 0)  // where the item's pieces are: its first one, and the CTA of its last
        p.pieces[(int64_t)w.b * p.heads_kv + kvh] = complete ? make_int2(-1, 0) : make_int2(part, (w.base + w.weight - 1) / share);
    }
    if (!next_piece<kTile>(p, w, stop)) break;
  }
}

template <pd_dtype T, int D, int NR, int H, int WK, int WR>
pd_status launch(const pd_paged_attention_desc& d, const Params& p, const Scales& scales, const void* k_cache, const void* v_cache,
                 cudaStream_t s) {
  using C = Q8Config<D, NR, H, WK, WR>;
  CUtensorMap tk, tv;
  const int box = d.page_size < C::kTile ? d.page_size : C::kTile;
  if (!make_cache_map_q8(&tk, k_cache, d, box, H) || !make_cache_map_q8(&tv, v_cache, d, box, H)) return PD_ERR_UNSUPPORTED;
  static PerDeviceFlag smem_allowed;
  if (pd_status st = allow_dynamic_smem(paged_attention_q8_rows_kernel<T, D, NR, H, WK, WR>, C::kSmem, smem_allowed); st != PD_OK) return st;
  launch_pdl(paged_attention_q8_rows_kernel<T, D, NR, H, WK, WR>, dim3(p.splits), dim3(kThreads), C::kSmem, s, tk, tv, p, scales);
  if (pd_status st = check_launch(); st != PD_OK || p.whole_items) return st;
  const int rows = (int)std::min<int64_t>((int64_t)p.max_q_len * p.group, C::kRows);
  const bool spread = (int64_t)d.heads_kv * d.batch * rows <= 4 * kSms;  // (more CTAs keep the loads coming)
  const dim3 grid(d.heads_kv, d.batch, spread ? rows : (rows + kJoinWarps - 1) / kJoinWarps);
  launch_pdl(paged_attention_join_rows<D>, grid, dim3(32 * kJoinWarps), 0, s, p, C::kRows, H, spread);
  return check_launch();
}
template <pd_dtype T, int D>
pd_status launch_plan(const pd_paged_attention_desc& d, const Params& p, const Plan& plan, const Scales& scales, const void* k, const void* v,
                      cudaStream_t s) {
  const int h = plan.heads_per_item;
  if (plan.rows_per_tile == 8)
    return h == 4 ? launch<T, D, 1, 4, 1, 1>(d, p, scales, k, v, s) : h == 2 ? launch<T, D, 1, 2, 2, 1>(d, p, scales, k, v, s) : launch<T, D, 1, 1, 4, 1>(d, p, scales, k, v, s);
  if (plan.rows_per_tile == 16)
    return h == 4 ? launch<T, D, 2, 4, 1, 1>(d, p, scales, k, v, s) : h == 2 ? launch<T, D, 2, 2, 2, 1>(d, p, scales, k, v, s) : launch<T, D, 2, 1, 4, 1>(d, p, scales, k, v, s);
  if (plan.rows_per_tile == 24)
    return h == 4 ? launch<T, D, 3, 4, 1, 1>(d, p, scales, k, v, s) : h == 2 ? launch<T, D, 3, 2, 2, 1>(d, p, scales, k, v, s) : launch<T, D, 3, 1, 4, 1>(d, p, scales, k, v, s);
  if (plan.rows_per_tile == 32)
    return h == 2 ? launch<T, D, 2, 2, 1, 2>(d, p, scales, k, v, s) : launch<T, D, 2, 1, 2, 2>(d, p, scales, k, v, s);
  return launch<T, D, 2, 1, 1, 4>(d, p, scales, k, v, s);
}

}  // namespace
}  // namespace paged
}  // namespace pd
