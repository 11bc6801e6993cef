// What the kernels of the paged attention for few rows per cache head share, whatever the cache's type: how the key tiles of
// all sequences and heads are dealt out to the CTAs, how a piece's partial results are written, and how the pieces of an item
// are joined.  Internal to the library.
#pragma once

#include "paged_cache.cuh"

namespace pd {
namespace paged {
namespace {

// One item, or a part of one: sequence and cache head (or group of them), its key tiles, and the tiles [begin, end) of `weight`
// that are meant.
struct Piece {
  Sequence seq;
  KeyTiles tiles;
  int b, kvh, rows;
  int weight;  // key tiles of the item; one at least where it has rows, so that somebody writes them
  int base;    // of the item, in the count of all tiles (the entry point bounds it)
  int begin, end;
};

template <int TILE>
__device__ __forceinline__ void set_sequence(const Params& p, int b, Piece& w) {
  w.b = b;
  w.seq = load_sequence(p, b);
  w.rows = w.seq.n * p.group;
  w.tiles = key_tiles(p, w.seq.pos0, w.seq.pos0 + w.seq.n - 1, w.seq.length, TILE);
  w.weight = w.rows > 0 ? max(w.tiles.n, 1) : 0;
}

// On to the next item; false when the share ends.
template <int TILE>
__device__ __forceinline__ bool next_piece(const Params& p, Piece& w, int stop) {
  w.base += w.weight;
  if (w.base >= stop) return false;
  if (++w.kvh == p.items) {
    w.kvh = 0;
    do set_sequence<TILE>(p, w.b + 1, w); while (w.weight == 0);  // (there is one: the share goes on)
  }
  w.begin = 0;
  w.end = p.whole_items ? w.weight : min(w.weight, stop - w.base);
  return true;
}

// The share of CTA `cta`: [start, stop) of all tiles, and in `w` the item that `start` lies in.  Collective over the block
// (THREADS threads); false if the share is empty.
template <int THREADS, int TILE>
__device__ __forceinline__ bool first_piece(const Params& p, int cta, Piece& w, int& start, int& stop, int& share) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int found_b, found_base, total;
  auto deal = [&]() {
    share = max((total + (int)gridDim.x - 1) / (int)gridDim.x, 1);
    const int64_t at = (int64_t)cta * share;
    start = (int)min(at, (int64_t)total);
    stop = (int)min(at + share, (int64_t)total);
    return start < stop;
  };
  auto scan = [&](int v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    return v;
  };
  if (p.batch <= 32) {  // every warp for itself
    int mine = 0;
    if (lane < p.batch) {
      set_sequence<TILE>(p, lane, w);
      mine = w.weight * p.items;
    }
    const int upto = scan(mine);
    total = __shfl_sync(0xffffffffu, upto, 31);
    if (!deal()) return false;
    found_b = __ffs(__ballot_sync(0xffffffffu, upto > start)) - 1;
    found_base = __shfl_sync(0xffffffffu, upto - mine, found_b);
  } else {  // a run of sequences per thread
    __shared__ int warp_sums[THREADS / 32], found[2];
    const int per = (p.batch + THREADS - 1) / THREADS, b0 = threadIdx.x * per;
    int mine = 0;
    for (int b = b0; b < min(b0 + per, p.batch); ++b) {
      set_sequence<TILE>(p, b, w);
      mine += w.weight * p.items;
    }
    int upto = scan(mine);
    if (lane == 31) warp_sums[warp] = upto;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) {
      if (k < warp) upto += warp_sums[k];
      total += warp_sums[k];
    }
    if (!deal()) return false;  // (uniform over the block)
    int base = upto - mine;
    if (base <= start && start < upto) {
      for (int b = b0;; ++b) {
        set_sequence<TILE>(p, b, w);
        const int next = base + w.weight * p.items;
        if (start < next) {
          found[0] = b;
          found[1] = base;
          break;
        }
        base = next;
      }
    }
    __syncthreads();
    found_b = found[0];
    found_base = found[1];
  }
  set_sequence<TILE>(p, found_b, w);
  w.kvh = (start - found_base) / w.weight;
  w.base = found_base + w.kvh * w.weight;
  w.begin = start - w.base;
  w.end = p.whole_items ? w.weight : min(w.weight, stop - w.base);
  // (whole items: they are the CTA's in whose share they begin)
  return !p.whole_items || w.begin == 0 || next_piece<TILE>(p, w, stop);
}

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Barrier of the consumer warps; true if any of their threads says so.
template <int THREADS>
__device__ __forceinline__ bool barrier_any(bool yes) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 q, %1, 0;\n"
      "bar.red.or.pred p, 1, %2, q;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(r)
      : "r"(yes ? 1u : 0u), "n"(THREADS)
      : "memory");
  return r != 0;
}

// The results of a piece: for every group of GROUP rows, PARTS partial results in `merge` (rows of D + 2 floats: the
// accumulator, the maximum in powers of two, the sum), which the consumer warps (THREADS) have written and published.  Rows of
// an item that is this CTA's alone go to the output, others to the workspace (tiles of ROWS rows).
template <int D, int GROUP, int PARTS, int ROWS, int THREADS>
__device__ __forceinline__ void write_piece(const Params& p, const Piece& w, int piece, int share, const float* merge) {
  constexpr int kStride = D + 2;
  const bool complete = w.begin == 0 && w.end == w.weight;
  const int part = 2 * blockIdx.x + (piece > 0 ? 1 : 0);  // a piece that is neither the CTA's first nor its last is complete
  // one group of D / 4 threads per row, four elements per thread
  constexpr int kPer = D / 4;
  for (int i = threadIdx.x; i < w.rows * kPer; i += THREADS) {
    const int r = i / kPer, d = (i % kPer) * 4;
    const float* part_r = merge + ((r / GROUP) * PARTS * GROUP + r % GROUP) * kStride;
    float mm = -INFINITY;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) mm = fmaxf(mm, part_r[k * GROUP * kStride + D]);
    float ll = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      const float* q = part_r + k * GROUP * kStride;
      const float f = q[D] == -INFINITY ? 0.f : ex2(q[D] - mm);
      ll += f * q[D + 1];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += f * q[d + j];
    }
    const float inv = ll > 0.f ? 1.f / ll : 0.f;  // nothing seen: zeros
    if (complete) {
      const int t = w.seq.q0 + r / p.group, h = w.kvh * p.group + r % p.group;
      uint2 v;
      v.x = pack_bf16(acc[0] * inv, acc[1] * inv);
      v.y = pack_bf16(acc[2] * inv, acc[3] * inv);
      *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.ld_out + (int64_t)h * D + d) = v;
    } else {
      const int64_t at = (int64_t)part * ROWS + r;
      if (ll > 0.f) *reinterpret_cast<float4*>(p.part_o + at * D + d) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
      if (d == 0) p.part_lse[at] = ll > 0.f ? mm + log2f(ll) : -INFINITY;
    }
  }
  if (threadIdx.x == 0 && w.begin == 0)  // where the item's pieces are: its first one, and the CTA of its last
    p.pieces[(int64_t)w.b * p.heads_kv + w.kvh] = complete ? make_int2(-1, 0) : make_int2(part, (w.base + w.weight - 1) / share);
}

// Joins the pieces of the items that several CTAs worked on: out = sum_z w_z O_z / sum_z w_z, w_z = 2^(lse_z - max lse).
// A CTA per item and eight of its rows, a warp per row; where there are fewer rows, several warps per row, which then take
// every so-manieth piece.
// Latency-bound: the loads of a warp's pieces are in flight together (one at a time, 37 pieces of a long context took 12 us).
constexpr int kJoinWarps = 8;
// `group`: cache heads to an item; their partial results lie behind one another.
// `spread`: the grid has a CTA for every row, which all of its warps work on where there are kSpread pieces and more.
//   (One sequence of 16384 keys, 4 cache heads, 8 rows, 256 pieces: 20 us for the call, with a warp to a row 41.  Joins of fewer pieces have
//   loads enough in flight either way: 16 sequences of 2048 keys, 16 rows, 18 pieces: 37 spread, 29 not.)
constexpr int kSpread = 32;
template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps) paged_attention_join_rows(const Params p, int rows_per_tile, int group, bool spread) {
  __shared__ float part[kJoinWarps][D + 2];
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.y, kvh = blockIdx.x;
  const int2 pieces = p.pieces[(int64_t)b * p.heads_kv + kvh];
  const Sequence seq = load_sequence(p, b);
  const int rows = seq.n * p.group;
  if (rows <= (int)blockIdx.z || pieces.x < 0) return;  // (no CTA had this item and wrote its entry; or one CTA had all of it)
  const int first_cta = pieces.x >> 1, n = pieces.y - first_cta + 1;
  const int rows_a_cta = spread && n >= kSpread ? 1 : kJoinWarps, r0 = blockIdx.z * rows_a_cta;
  if (rows <= r0) return;
  // (a CTA whose wait for a key tile ran out has left the entry as it was in the workspace)
  if (first_cta >= p.splits || pieces.y >= p.splits || pieces.y < first_cta) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int per_row = 1;
  while (2 * per_row * min(rows, rows_a_cta) <= kJoinWarps) per_row *= 2;
  constexpr int kCols = D / 32;
  {
    const int r = r0 + warp / per_row, z0 = warp % per_row;
    auto at = [&](int z) { return ((int64_t)(z == 0 ? pieces.x : 2 * (first_cta + z)) * group + kvh % group) * rows_per_tile + r; };
    float top = -INFINITY, sum = 0.f, acc[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
    if (r < rows) {
      for (int z = lane; z < n; z += 32) top = fmaxf(top, p.part_lse[at(z)]);
      for (int base = z0; base < n; base += 8 * per_row) {
        float lse[8], o[8][kCols];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int z = base + k * per_row;
          lse[k] = z < n ? p.part_lse[at(z)] : -INFINITY;
          const float* src = p.part_o + at(min(z, n - 1)) * D + lane * kCols;
#pragma unroll
          for (int j = 0; j < kCols; ++j) o[k][j] = src[j];
        }
        if (base == z0) top = warp_max(top);  // (here, so that the first loads are under way)
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (lse[k] > -INFINITY) {  // (a piece that saw nothing has left its output unwritten)
            const float f = ex2(lse[k] - top);
            sum += f;
#pragma unroll
            for (int j = 0; j < kCols; ++j) acc[j] = fmaf(f, o[k][j], acc[j]);
          }
      }
    }
    if (per_row > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kCols; ++j) part[warp][lane * kCols + j] = acc[j];
      if (lane == 0) part[warp][D] = sum;
      __syncthreads();
      if (z0 == 0)
        for (int k = 1; k < per_row; ++k) {
          sum += part[warp + k][D];
#pragma unroll
          for (int j = 0; j < kCols; ++j) acc[j] += part[warp + k][lane * kCols + j];
        }
    }
    if (r < rows && z0 == 0) {
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      const int t = seq.q0 + r / p.group, h = kvh * p.group + r % p.group;
      uint32_t* out = reinterpret_cast<uint32_t*>(p.out + (int64_t)t * p.ld_out + (int64_t)h * D + lane * kCols);
#pragma unroll
      for (int j = 0; j < kCols; j += 2) out[j / 2] = pack_bf16(acc[j] * inv, acc[j + 1] * inv);
    }
  }
}

}  // namespace
}  // namespace paged
}  // namespace pd
