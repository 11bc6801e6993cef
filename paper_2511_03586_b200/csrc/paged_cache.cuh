// Pieces shared by the kernels that write and read the paged key/value cache: which sequence a token belongs to,
// which keys the rows of a tile see, in which key tiles these lie, and the tensor maps of the caches.
// Internal to the library.
#pragma once

#include "gemm_common.cuh"

namespace pd {
namespace paged {

using namespace sm100;

// Kernel parameters of the attention over the cache.  A "row" is one (token, query head) pair of one cache head:
// row r of sequence b and cache head k stands for its token r / group and its query head k * group + r % group, so
// that the query heads that share keys share the tile that reads them.
struct Params {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const int32_t *block_table, *cu_q, *kv_len;
  // Partial outputs (normalised) and the logarithms (base 2) of their sums of exponentials: [splits][part_tokens * heads_q]
  // (chunk kernel), or [2 CTAs][rows per tile] with the places of an item's pieces (row kernel).
  float *part_o, *part_lse;
  int2* pieces;
  int* status;
  unsigned long long wait_limit_ns;  // of every bounded wait
  int withhold_loads;                // test switch: key tiles are not requested, and the first wait for one runs out
  int64_t ld_q, ld_out;
  int batch, tokens, heads_q, heads_kv, group;
  int num_pages, page_size, page_shift, max_pages;
  int max_q_len, window, sinks;
  // Tokens that can have partial results in the chunk kernel: all rows of the token tensors, or, where these are padded to
  // more than max_q_len for each sequence, that many places a sequence.
  int part_tokens, part_by_sequence;
  int splits;           // of the keys of every row tile (chunk kernel), CTAs in all (row kernel)
  int min_split_tiles;  // the smallest share of key tiles (chunk kernel)
  int whole_items;      // row kernel: no item is shared out (short contexts: nothing to join)
  float scale_log2e;
};

// Codes left in the device status word by an expired wait.
enum : int { kTimeoutRowsProducer = 301, kTimeoutRowsConsumer = 302, kTimeoutChunkProducer = 311, kTimeoutChunkMma = 312,
             kTimeoutChunkSoftmax = 313 };

// The number of entries cu[1 ... n] that are <= t (they ascend): the sequence that token t belongs to, n if none.
__device__ __forceinline__ int find_sequence(const int32_t* cu, int n, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;  // the answer lies in [lo, hi]
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const int i = lo + lane * step;  // is entry i + 1 <= t ?
    const unsigned le = __ballot_sync(0xffffffffu, i < hi && __ldg(cu + i + 1) <= t);
    const int k = __popc(le);  // probes lo, lo + step, ..., lo + (k - 1) step are <= t, the next one is not
    if (k == 0) return lo;
    const int next = lo + (k - 1) * step + 1;
    hi = min(lo + k * step, hi);
    lo = next;
  }
  return lo;
}

struct Sequence {
  int q0, n;     // first token row, new tokens (as many as are computed)
  int pos0;      // position of the first new token (negative when kv_len is short of n)
  int length;    // keys that the block table can name
  int part0;     // place of the first token's partial results
};

__device__ __forceinline__ Sequence load_sequence(const Params& p, int b) {
  Sequence s;
  const int a = min(max(__ldg(p.cu_q + b), 0), p.tokens);
  const int e = min(max(__ldg(p.cu_q + b + 1), a), p.tokens);
  const int64_t cap = (int64_t)p.max_pages << p.page_shift;
  const int len = max(__ldg(p.kv_len + b), 0);
  s.q0 = a;
  s.n = min(e - a, p.max_q_len);
  s.pos0 = len - (e - a);
  s.length = (int)(len < cap ? len : cap);
  s.part0 = p.part_by_sequence ? b * p.max_q_len : a;
  return s;
}

// The key tiles of `tile` keys that some of the positions first ... last sees: the tiles of the sink tokens, then
// those from the first position's window to the last position; [sink_hi, lo) is in nobody's view.
struct KeyTiles {
  int lo, hi;      // keys in the view of some window: [lo, hi)
  int sink_hi;     // keys in view as sinks: [0, sink_hi)
  int n_sink;      // tiles taken from the sinks
  int first;       // first tile of the window part
  int n;           // tiles in all
  __device__ __forceinline__ int tile_index(int i) const { return i < n_sink ? i : first + (i - n_sink); }
};

__device__ __forceinline__ KeyTiles key_tiles(const Params& p, int first_pos, int last_pos, int length, int tile) {
  KeyTiles t;
  t.hi = max(min(last_pos + 1, length), 0);
  t.lo = p.window > 0 ? min(max(first_pos - p.window + 1, 0), t.hi) : 0;
  t.sink_hi = p.window > 0 ? min(p.sinks, t.hi) : 0;
  const int end = (t.hi + tile - 1) / tile;
  t.first = t.lo / tile;
  t.n_sink = min((t.sink_hi + tile - 1) / tile, t.first);  // tiles that the window part does not hold anyway
  t.n = t.hi > 0 ? t.n_sink + end - t.first : 0;
  return t;
}

// The share [begin, end) of split `z` in `n` key tiles: even shares, but none below min_split_tiles, so that short
// sequences of a ragged batch leave their last splits empty instead of cutting themselves to pieces.
__device__ __forceinline__ void split_range(const Params& p, int n, int z, int& begin, int& end) {
  const int per = max((n + p.splits - 1) / p.splits, p.min_split_tiles);
  begin = min(z * per, n);
  end = min(begin + per, n);
}

// Page of the cache that holds key `key` of sequence b, or num_pages (out of range: TMA fills with zeros) where the
// table has no such page.
__device__ __forceinline__ int page_of(const Params& p, int b, int key) {
  const int i = key >> p.page_shift;
  if (i >= p.max_pages) return p.num_pages;
  const int e = __ldg(p.block_table + (int64_t)b * p.max_pages + i);
  return (unsigned)e < (unsigned)p.num_pages ? e : p.num_pages;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// ---- host side -----------------------------------------------------------------------
// Tensor map of one cache: {head_dim, page_size, heads_kv, num_pages}, boxes of 64 elements x `box_rows` slots.
inline bool make_cache_map(CUtensorMap* map, const void* cache, const pd_paged_attention_desc& d, int box_rows) {
  gemm::EncodeTiledFn fn = gemm::encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)d.head_dim, (cuuint64_t)d.page_size, (cuuint64_t)d.heads_kv,
                              (cuuint64_t)d.num_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)d.slot_stride * 2, (cuuint64_t)d.head_stride * 2,
                                 (cuuint64_t)d.page_stride * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(cache), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Launchers (each in its own file).  `rows_per_tile` of the row kernel: 16, 32 or 64.
pd_status launch_rows(const pd_paged_attention_desc& d, Params& p, const void* k_cache, const void* v_cache,
                      int rows_per_tile, cudaStream_t s);
pd_status launch_chunk(const pd_paged_attention_desc& d, const Params& p, const void* k_cache, const void* v_cache,
                       cudaStream_t s);

}  // namespace paged
}  // namespace pd
