// Attention over the paged cache for few rows per cache head (single tokens, drafts, short chunks):
//
//   out[t, h] = sum_j softmax_j(scale * q[t, h] . k[j]) v[j],   j visible from token t's position
//
// Bound: HBM. Every key and value in view is read once per tile of 16 to 64 rows, and a row takes 4 D flops per key, so
// that with 16 rows the arithmetic is 16 flops per byte: mma.sync on register fragments keeps up with memory several
// times over, and leaves tensor memory and its hand-overs out of a kernel that waits for loads.
//
// A CTA takes one tile of rows of one cache head and one share of its keys.  A producer warp looks the pages up and
// copies key tiles of 64 keys with TMA, one box per page, into a ring of stages (128-byte swizzle, which makes ldmatrix
// conflict-free); two CTAs per SM with 96 KiB each keep about 130 KiB of copies in flight per SM.  The consumer warps
// are WR x WK: WR groups of 16 rows, and within a group WK warps that take 64 / WK keys of every tile each, with a
// running maximum and sum of their own; nothing is exchanged before the end, where the WK partial results meet in
// shared memory.  With `splits` > 1 the CTAs of a row tile take even shares of the keys and leave normalised partial
// outputs and log-sum-exps in the workspace, which paged_attention_join joins.
#include "paged_cache.cuh"

namespace pd {
namespace paged {
namespace {

constexpr int kTile = 64;  // keys per stage
constexpr int kRing = 96 * 1024;

template <int D, int WR, int WK>
struct RowsConfig {
  static constexpr int kRows = 16 * WR;
  static constexpr int kConsumers = WR * WK;
  static constexpr int kThreads = 32 * (kConsumers + 1);
  static constexpr int kTensorBytes = kTile * D * 2;     // K or V of a stage
  static constexpr int kStageBytes = 2 * kTensorBytes;
  static constexpr int kStages = kRing / kStageBytes;
  static constexpr int kSmem = kRing + 1024 /*barriers*/ + 1024 /*alignment*/;
  static constexpr int kMergeStride = D + 2;             // floats per row of a warp's partial result: O, m, l
  static_assert(kConsumers * 16 * kMergeStride * 4 <= kRing, "the partial results fit into the drained ring");
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D, int WR, int WK>
__global__ void __launch_bounds__(RowsConfig<D, WR, WK>::kThreads, 2)
paged_attention_rows_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                            const Params p) {
  using C = RowsConfig<D, WR, WK>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  float* merge = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw)));
  const uint32_t bars = ring + kRing;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 128u + 8u * s; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + (bars - smem_u32(smem_raw)) + 256);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), C::kConsumers); }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == C::kConsumers && lane == 0) { prefetch_tensormap(&tmap_k); prefetch_tensormap(&tmap_v); }
  __syncthreads();
  griddep_wait();
  griddep_launch_dependents();

  const int split = blockIdx.x % p.splits, row_tile = blockIdx.x / p.splits;
  const int kvh = blockIdx.y, b = blockIdx.z;
  const Sequence seq = load_sequence(p, b);
  const int row0 = row_tile * C::kRows;
  const int rows = min(seq.n * p.group - row0, C::kRows);
  if (rows <= 0) return;
  const int first_pos = seq.pos0 + row0 / p.group, last_pos = seq.pos0 + (row0 + rows - 1) / p.group;
  const KeyTiles kt = key_tiles(p, first_pos, last_pos, seq.length, kTile);
  int begin, end;
  split_range(p, kt.n, split, begin, end);

  if (warp == C::kConsumers) {
    // ------------------------------------------------------------------ producer
    // Per stage: 64 / page_size pages (or a part of one), each a box of `box` slots by 64 elements.  The lanes hold
    // the pages of the next `per_batch` tiles.
    const int box = min(p.page_size, kTile);
    const int per_tile = kTile / box;
    const int per_batch = 32 / per_tile;
    int page = 0;
    bool ok = true;
    int it = 0;
    for (int i = begin; i < end; ++i, ++it) {
      const int in_batch = it % per_batch;
      if (in_batch == 0) {
        const int ti = i + lane / per_tile;
        page = ti < end ? page_of(p, b, kt.tile_index(ti) * kTile + (lane % per_tile) * box) : 0;
      }
      const int stage = it % C::kStages;
      if (!mbar_wait_warp(empty(stage), ((it / C::kStages) & 1u) ^ 1u, abort_flag, p.status, kTimeoutRowsProducer)) { ok = false; break; }
      const uint32_t k_dst = ring + stage * C::kStageBytes, v_dst = k_dst + C::kTensorBytes;
      const int slot = (kt.tile_index(i) * kTile) & (p.page_size - 1);  // 0 unless a page holds several tiles
      if (elect_one()) mbar_arrive_expect_tx(full(stage), C::kStageBytes);
      __syncwarp();
      for (int j = 0; j < per_tile; ++j) {
        const int pg = __shfl_sync(0xffffffffu, page, in_batch * per_tile + j);
        if (elect_one()) {
#pragma unroll
          for (int h = 0; h < D / 64; ++h) {
            const uint32_t at = (uint32_t)(h * kTile + j * box) * 128u;
            tma_load_4d(k_dst + at, &tmap_k, full(stage), h * 64, slot, kvh, pg);
            tma_load_4d(v_dst + at, &tmap_v, full(stage), h * 64, slot, kvh, pg);
          }
        }
        __syncwarp();
      }
    }
    if (!ok) {
      // leave no copy in flight: give the last request of every stage a short time to land
      volatile int never = 0;
      for (int back = 1; back <= C::kStages && back <= it; ++back) {
        const int i = it - back;
        mbar_wait(full(i % C::kStages), (i / C::kStages) & 1u, &never, nullptr, 0, 20000000ull);
      }
    }
    return;
  }

  // ------------------------------------------------------------------- consumers
  const int wr = warp / WK, wk = warp % WK;
  constexpr int kKeys = kTile / WK;  // keys of a tile that are this warp's
  constexpr int NT = kKeys / 8, KS = D / 16;
  // rows of this lane in the fragments: g and g + 8 of the warp's 16
  const int g = lane >> 2, c2 = (lane & 3) * 2;
  uint32_t qf[KS][4];
  int pos[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = wr * 16 + g + 8 * i;
    const int rr = row0 + min(r, rows - 1);
    const int t = rr / p.group;
    pos[i] = seq.pos0 + t;  // (rows beyond the last repeat it and are not stored)
    const __nv_bfloat16* qr = p.q + (int64_t)(seq.q0 + t) * p.ld_q + (int64_t)(kvh * p.group + rr % p.group) * D;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      qf[k][i] = __ldg(reinterpret_cast<const uint32_t*>(qr + 16 * k + c2));
      qf[k][2 + i] = __ldg(reinterpret_cast<const uint32_t*>(qr + 16 * k + 8 + c2));
    }
  }
  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};  // maximum (in units of the base-2 exponent), this lane's part of the sum

  // shared-memory addresses of this lane's ldmatrix rows, relative to the stage
  const int k_row = (lane & 7) + ((lane >> 4) << 3);   // K: matrices (keys 0-7, d 0-7), (0-7, 8-15), (8-15, 0-7), (8-15, 8-15)
  const int k_chunk = (lane >> 3) & 1;
  const int v_row = lane & 15, v_chunk = lane >> 4;    // V: (keys 0-7, d 0-7), (8-15, 0-7), (0-7, d 8-15), (8-15, 8-15)

  int it = 0;
  for (int i = begin; i < end; ++i, ++it) {
    const int stage = it % C::kStages;
    // (a warp that gives up has raised the flag: it goes on to the barriers below, behind which nothing is stored)
    if (!mbar_wait_warp(full(stage), (it / C::kStages) & 1u, abort_flag, p.status, kTimeoutRowsConsumer)) break;
    const uint32_t sk = ring + stage * C::kStageBytes, sv = sk + C::kTensorBytes;
    const int key0 = kt.tile_index(i) * kTile + wk * kKeys;
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int n2 = 0; n2 < NT / 2; ++n2) {
      const int row = wk * kKeys + n2 * 16 + k_row;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t kf[4];
        ldmatrix_x4(sk + (uint32_t)((k >> 2) * kTile + row) * 128u + ((uint32_t)(((k & 3) * 2 + k_chunk) ^ (row & 7)) << 4), kf);
        mma_16816(s[2 * n2], qf[k], kf[0], kf[1]);
        mma_16816(s[2 * n2 + 1], qf[k], kf[2], kf[3]);
      }
    }
    // keys outside a row's view; whole tiles in everybody's view skip this
    const int last_key = key0 + kKeys - 1;
    const bool whole = last_key <= first_pos && last_key < seq.length &&
                       (p.window == 0 || key0 > last_pos - p.window || last_key < p.sinks);
    if (!whole) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = key0 + n * 8 + c2 + (e & 1), at = pos[e >> 1];
          const bool seen = key <= at && key < seq.length && (p.window == 0 || key > at - p.window || key < p.sinks);
          if (!seen) s[n][e] = -INFINITY;
        }
    }
    float ref[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float mx = -INFINITY;
#pragma unroll
      for (int n = 0; n < NT; ++n) mx = fmaxf(mx, fmaxf(s[n][2 * e], s[n][2 * e + 1]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      ref[e] = fmaxf(m[e], mx * p.scale_log2e);
    }
    if (__any_sync(0xffffffffu, ref[0] > m[0] || ref[1] > m[1])) {
      const float a0 = ref[0] > m[0] ? ex2(m[0] - ref[0]) : 1.f, a1 = ref[1] > m[1] ? ex2(m[1] - ref[1]) : 1.f;
      l[0] *= a0; l[1] *= a1;
#pragma unroll
      for (int d = 0; d < D / 8; ++d) { o[d][0] *= a0; o[d][1] *= a0; o[d][2] *= a1; o[d][3] *= a1; }
      m[0] = ref[0]; m[1] = ref[1];
    }
    // a row that has seen nothing yet is referred to 0: its exponentials are 2^-inf = 0
    const float r0 = ref[0] == -INFINITY ? 0.f : ref[0], r1 = ref[1] == -INFINITY ? 0.f : ref[1];
    uint32_t pf[NT / 2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float e0 = ex2(fmaf(s[n][0], p.scale_log2e, -r0)), e1 = ex2(fmaf(s[n][1], p.scale_log2e, -r0));
      const float e2 = ex2(fmaf(s[n][2], p.scale_log2e, -r1)), e3 = ex2(fmaf(s[n][3], p.scale_log2e, -r1));
      l[0] += e0 + e1; l[1] += e2 + e3;
      pf[n >> 1][(n & 1) * 2] = pack_bf16(e0, e1);
      pf[n >> 1][(n & 1) * 2 + 1] = pack_bf16(e2, e3);
    }
#pragma unroll
    for (int k = 0; k < kKeys / 16; ++k) {
      const int row = wk * kKeys + k * 16 + v_row;
      // Values of keys in nobody's view may hold anything: zeroed, since 0 * NaN is NaN.  b0 holds keys c2, c2 + 1 of
      // the step, b1 the keys 8 further.
      uint32_t mask0 = 0xffffffffu, mask1 = 0xffffffffu;
      if (!whole) {
        auto half = [&](int key) { return (key < kt.hi && key >= kt.lo) || key < kt.sink_hi ? 0xffffu : 0u; };
        const int key = key0 + k * 16 + c2;
        mask0 = half(key) | half(key + 1) << 16;
        mask1 = half(key + 8) | half(key + 9) << 16;
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        uint32_t vf[4];
        ldmatrix_x4_trans(sv + (uint32_t)((d >> 2) * kTile + row) * 128u + ((uint32_t)(((d & 3) * 2 + v_chunk) ^ (row & 7)) << 4), vf);
        if (!whole) { vf[0] &= mask0; vf[1] &= mask1; vf[2] &= mask0; vf[3] &= mask1; }
        mma_16816(o[2 * d], pf[k], vf[0], vf[1]);
        mma_16816(o[2 * d + 1], pf[k], vf[2], vf[3]);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty(stage));
  }

#pragma unroll
  for (int e = 0; e < 2; ++e) {
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
    l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
  }
  // the ring has been read by every warp; the partial results take its place
  asm volatile("bar.sync 1, %0;" ::"n"(32 * C::kConsumers) : "memory");
  float* mine = merge + (wr * WK + wk) * 16 * C::kMergeStride;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    float* row = mine + (g + 8 * e) * C::kMergeStride;
#pragma unroll
    for (int d = 0; d < D / 8; ++d) *reinterpret_cast<float2*>(row + d * 8 + c2) = make_float2(o[d][2 * e], o[d][2 * e + 1]);
    if ((lane & 3) == 0) { row[D] = m[e]; row[D + 1] = l[e]; }
  }
  asm volatile("bar.sync 1, %0;" ::"n"(32 * C::kConsumers) : "memory");
  if (*abort_flag) return;
  // one group of D / 4 threads per row, four elements per thread
  constexpr int kPer = D / 4;
  for (int i = threadIdx.x; i < rows * kPer; i += 32 * C::kConsumers) {
    const int r = i / kPer, d = (i % kPer) * 4;
    const float* part = merge + ((r / 16) * WK * 16 + r % 16) * C::kMergeStride;
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < WK; ++w) mm = fmaxf(mm, part[w * 16 * C::kMergeStride + D]);
    float ll = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float* q = part + w * 16 * C::kMergeStride;
      const float f = q[D] == -INFINITY ? 0.f : ex2(q[D] - mm);
      ll += f * q[D + 1];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += f * q[d + j];
    }
    const float inv = ll > 0.f ? 1.f / ll : 0.f;  // nothing seen: zeros
    const int rr = row0 + r, t = seq.q0 + rr / p.group, h = kvh * p.group + rr % p.group;
    if (p.splits == 1) {
      uint2 w;
      w.x = pack_bf16(acc[0] * inv, acc[1] * inv);
      w.y = pack_bf16(acc[2] * inv, acc[3] * inv);
      *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.ld_out + (int64_t)h * D + d) = w;
    } else {
      const int64_t at = ((int64_t)split * p.tokens + t) * p.heads_q + h;
      if (ll > 0.f) *reinterpret_cast<float4*>(p.part_o + at * D + d) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
      if (d == 0) p.part_lse[at] = ll > 0.f ? mm + log2f(ll) : -INFINITY;
    }
  }
}

template <int D, int WR, int WK>
pd_status launch(const pd_paged_attention_desc& d, const Params& p, const CUtensorMap& tk, const CUtensorMap& tv,
                 cudaStream_t s) {
  using C = RowsConfig<D, WR, WK>;
  static PerDeviceFlag smem_allowed;
  if (pd_status st = allow_dynamic_smem(paged_attention_rows_kernel<D, WR, WK>, C::kSmem, smem_allowed); st != PD_OK) return st;
  const int64_t row_tiles = ((int64_t)p.max_q_len * p.group + C::kRows - 1) / C::kRows;
  if (row_tiles * p.splits > 0x7fffffff) return PD_ERR_BAD_SHAPE;
  launch_pdl(paged_attention_rows_kernel<D, WR, WK>, dim3((unsigned)(row_tiles * p.splits), d.heads_kv, d.batch),
             dim3(C::kThreads), C::kSmem, s, tk, tv, p);
  return check_launch();
}

}  // namespace

pd_status launch_rows(const pd_paged_attention_desc& d, Params& p, const void* k_cache, const void* v_cache,
                      int rows_per_tile, cudaStream_t s) {
  CUtensorMap tk, tv;
  const int box = d.page_size < kTile ? d.page_size : kTile;
  if (!make_cache_map(&tk, k_cache, d, box) || !make_cache_map(&tv, v_cache, d, box)) return PD_ERR_UNSUPPORTED;
  if (d.head_dim == 64) {
    if (rows_per_tile == 16) return launch<64, 1, 4>(d, p, tk, tv, s);
    if (rows_per_tile == 32) return launch<64, 2, 2>(d, p, tk, tv, s);
    return launch<64, 4, 1>(d, p, tk, tv, s);
  }
  if (rows_per_tile == 16) return launch<128, 1, 4>(d, p, tk, tv, s);
  if (rows_per_tile == 32) return launch<128, 2, 2>(d, p, tk, tv, s);
  return launch<128, 4, 1>(d, p, tk, tv, s);
}

}  // namespace paged
}  // namespace pd
