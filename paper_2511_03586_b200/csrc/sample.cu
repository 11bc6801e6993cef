// One token per row of logits under temperature, top-k, top-p and min-p, from a given random number:
//
//   w[j] = exp((logits[j] - max) / T), ranked by logit, then by index; keep the first top_k, of these the shortest
//   leading run that reaches top_p of their weight, of these the ones with w >= min_p; draw the first index at which
//   the running kept weight exceeds u times its total.
//
// Nothing is sorted.  Both cuts are "the first rank at which a running sum reaches a target", which a histogram by value
// finds: bin, sum the bins in descending order, and look again inside the bin that crosses, until a bin is a single
// logit value; of equal logits the first few by index are kept.
//
// Weights are summed as integers in units of 2^-44 of the largest weight (a row of 327680 weights stays below 2^63).
// Integer sums do not depend on their order, so atomics and any split over threads give the same bits, and the border of
// a cut, which decides between two tokens, is where the 64-bit definition has it: the exponential is evaluated in double
// precision (2^(n/64) from a table, the rest by its Taylor series to the fifth power: (ln 2 / 128)^6 / 6! < 2^-53).
//
// HBM-bound in principle: the logits are read once, 4 (or 2) bytes each, and held in the shared memory of a cluster of
// 1 to 8 CTAs (distributed by contiguous slices, so that index order is slice order).  In fact the passes over shared
// memory, the double-precision exponentials (eleven operations each) and the histogram's atomics weigh as much.
#include <cooperative_groups.h>

#include <cmath>

#include "pd_common.cuh"

namespace pd {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 1024;
constexpr float kBinsPerUnit = 32.f;  // first level: bins of 1/32 in z = (max - logit) / T, up to z = 32 (weight 2^-46: zero units)
constexpr int kFixed = 44;            // weights in units of 2^-44
constexpr int kMaxCluster = 8;
constexpr int64_t kMaxVocab = 327680;  // 8 slices of 160 KiB

using u64 = unsigned long long;

struct SampleParams {
  const void* logits;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* tokens;
  float* probs;
  int64_t ld;
  int vocab, slice;  // slice: logits per CTA, a multiple of 8
};

// Order-reversing map of floats to integers: larger logits have smaller keys.  (-0 has been made +0, NaN -inf.)
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v);
  return ~(b ^ ((b & 0x80000000u) ? 0xffffffffu : 0x80000000u));
}
__device__ __forceinline__ float value_of(uint32_t key) {
  const uint32_t a = ~key;
  return __uint_as_float((a & 0x80000000u) ? a ^ 0x80000000u : ~a);
}

struct Row {
  float max;
  double inv_t;      // 1 / T
  float bin_scale;   // kBinsPerUnit / T
  const double* table;
  // weight of logit v in units of 2^-44
  __device__ __forceinline__ u64 weight(float v) const {
    if (v == max) return 1ull << kFixed;
    const double x = ((double)v - (double)max) * inv_t;
    if (!(x > -32.0)) return 0;  // also max = +inf, and -inf logits
    constexpr double kLn2 = 0.69314718055994530942;
    constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits hold the rounded integer
    const double y = x * (64.0 / kLn2);
    const double r = y + kMagic;
    const int n = (int)__double2loint(r);
    constexpr double c = kLn2 / 64.0;
    const double f = y - (r - kMagic);
    double q = fma(c * c * c * c * c / 120.0, f, c * c * c * c / 24.0);
    q = fma(q, f, c * c * c / 6.0);
    q = fma(q, f, c * c / 2.0);
    q = fma(q, f, c);
    q = fma(q, f, 1.0);
    q *= table[n & 63];                                                         // in [0.99, 2)
    q = __hiloint2double(__double2hiint(q) + (((n >> 6) + kFixed) << 20), __double2loint(q));  // times 2^(n / 64 + 44)
    const double whole = q + 4503599627370496.0;                               // 2^52: rounds to an integer
    return (u64)__double_as_longlong(whole) & ((1ull << 52) - 1);
  }
  // first-level bin: a monotone function of v (each rounding is monotone); kBins for weights of zero
  __device__ __forceinline__ int bin(float v) const {
    if (v == max) return 0;
    const float t = (max - v) * bin_scale;
    return t < (float)kBins ? (int)t : kBins;
  }
};

struct Shared {
  double table[64];
  // own histogram, then the cluster's sums of the bins this CTA owns (first level, later levels)
  uint32_t count[kBins], lo[kBins], hi[kBins];
  uint32_t sum_count[2][kBins];
  u64 sum_weight[2][kBins];
  // published to the cluster
  u64 slice_weight[2];
  uint32_t slice_count[2];
  u64 above_weight;
  uint32_t equal_count;
  float row_max;
  // scratch of one CTA
  u64 warp_weight[kWarps];
  uint32_t warp_count[kWarps];
  float warp_max[kWarps];
  // result of a search step
  int found_bin;
  u64 found_weight_before, found_weight;
  uint32_t found_count_before, found_count;
  uint32_t range[2];
};

__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ u64 warp_scan_u64(u64 v) {  // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 w = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += w;
  }
  return v;
}
__device__ __forceinline__ uint32_t warp_scan_u32(uint32_t v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t w = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += w;
  }
  return v;
}

// Adds one logit to the own histogram: its weight in two 32-bit halves with the carry between them passed on by hand
// (shared memory has no native 64-bit addition).
__device__ __forceinline__ void add_to_bin(Shared& sh, int b, u64 w) {
  atomicAdd(&sh.count[b], 1u);
  const uint32_t lo = (uint32_t)w;
  const uint32_t before = atomicAdd(&sh.lo[b], lo);
  const uint32_t hi = (uint32_t)(w >> 32) + (before + lo < before ? 1u : 0u);
  if (hi) atomicAdd(&sh.hi[b], hi);
}

// Sums the cluster's histograms: CTA r gets the bins [r, r + 1) * kBins / n, and every CTA the sums over these slices of
// bins.  `level` 0 keeps the sums of the first histogram for a second search.
__device__ void sum_bins(cg::cluster_group& cluster, Shared& sh, int level, int n, int rank) {
  cluster.sync();  // every histogram is complete
  const int own = kBins / n;
  u64 tw = 0;
  uint32_t tc = 0;
  for (int i = threadIdx.x; i < own; i += kThreads) {
    const int b = rank * own + i;
    u64 w = 0;
    uint32_t c = 0;
    for (int r = 0; r < n; ++r) {
      const Shared* peer = cluster.map_shared_rank(&sh, r);
      c += peer->count[b];
      w += ((u64)peer->hi[b] << 32) + peer->lo[b];
    }
    sh.sum_count[level][i] = c;
    sh.sum_weight[level][i] = w;
    tw += w;
    tc += c;
  }
  tw = warp_sum_u64(tw);
  tc = __reduce_add_sync(0xffffffffu, tc);
  if ((threadIdx.x & 31) == 0) { sh.warp_weight[threadIdx.x >> 5] = tw; sh.warp_count[threadIdx.x >> 5] = tc; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWarps; ++w) { tw += sh.warp_weight[w]; tc += sh.warp_count[w]; }
    sh.slice_weight[level] = tw;
    sh.slice_count[level] = tc;
  }
  cluster.sync();  // the sums can be read, and nobody reads the histograms any more
}

// Finds the first bin at which the running count (by_count) or weight reaches `target`, and leaves it in sh.found_*; the
// last non-empty bin when the total stays below.  Collective over the CTA; every CTA of the cluster finds the same.
__device__ void find_bin(cg::cluster_group& cluster, Shared& sh, int level, int n, bool by_count, u64 target) {
  const int own = kBins / n;
  __syncthreads();  // the previous search's result and scratch have been read
  u64 before_w = 0;
  uint32_t before_c = 0;
  int owner = -1;
  u64 w0 = 0;
  uint32_t c0 = 0;
  for (int r = 0; r < n; ++r) {
    const Shared* peer = cluster.map_shared_rank(&sh, r);
    const u64 w = peer->slice_weight[level];
    const uint32_t c = peer->slice_count[level];
    if (c > 0) {
      owner = r;
      w0 = before_w;
      c0 = before_c;
    }
    before_w += w;
    before_c += c;
    if (owner == r && (by_count ? (u64)before_c : before_w) >= target) break;
  }
  const Shared* peer = cluster.map_shared_rank(&sh, owner < 0 ? 0 : owner);
  // thread i takes `per` consecutive bins of the owner's slice
  const int per = (own + kThreads - 1) / kThreads;
  u64 w[kBins / kThreads], tw = 0;
  uint32_t c[kBins / kThreads], tc = 0;
#pragma unroll
  for (int j = 0; j < kBins / kThreads; ++j) {
    const int i = threadIdx.x * per + j;
    const bool in = j < per && i < own;
    w[j] = in ? peer->sum_weight[level][i] : 0;
    c[j] = in ? peer->sum_count[level][i] : 0;
    tw += w[j];
    tc += c[j];
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  u64 sw = warp_scan_u64(tw);
  uint32_t sc = warp_scan_u32(tc);
  if (lane == 31) { sh.warp_weight[warp] = sw; sh.warp_count[warp] = sc; }
  if (threadIdx.x == 0) sh.found_bin = -1;
  __syncthreads();
  for (int k = 0; k < warp; ++k) { sw += sh.warp_weight[k]; sc += sh.warp_count[k]; }
  u64 rw = w0 + sw - tw;
  uint32_t rc = c0 + sc - tc;
  // candidate bins: every non-empty bin whose predecessor sum is below the target; the last of them is the answer
#pragma unroll
  for (int j = 0; j < kBins / kThreads; ++j) {
    if (c[j] > 0 && (by_count ? (u64)rc : rw) < target) atomicMax(&sh.found_bin, (int)threadIdx.x * per + j);
    rw += w[j];
    rc += c[j];
  }
  __syncthreads();
  rw = w0 + sw - tw;
  rc = c0 + sc - tc;
#pragma unroll
  for (int j = 0; j < kBins / kThreads; ++j) {
    if (j < per && sh.found_bin == (int)threadIdx.x * per + j) {
      sh.found_weight_before = rw;
      sh.found_count_before = rc;
      sh.found_weight = w[j];
      sh.found_count = c[j];
    }
    rw += w[j];
    rc += c[j];
  }
  __syncthreads();
  const int found = sh.found_bin;
  __syncthreads();
  if (threadIdx.x == 0) sh.found_bin = found + (owner < 0 ? 0 : owner) * own;
  __syncthreads();
}

// The cut: logits with a smaller key are kept, of those with this key the first `ties` by index.
struct Cut {
  uint32_t key;
  uint32_t ties;
  u64 weight;  // of everything kept
};

// First level already in sh.sum_*[0]: descends to the single logit value at which the running count or weight reaches
// `target`.
__device__ Cut search(cg::cluster_group& cluster, Shared& sh, const Row& row, const float* vals, int len, int n, int rank,
                      bool by_count, u64 target) {
  find_bin(cluster, sh, 0, n, by_count, target);
  u64 weight_before = sh.found_weight_before;
  uint32_t count_before = sh.found_count_before;
  // the keys of the bin: [first key with bin >= b, first key with bin >= b + 1), by bisection
  if (threadIdx.x < 2) {
    const int b = sh.found_bin + (int)threadIdx.x;
    uint32_t lo = key_of(row.max), hi = key_of(-INFINITY);
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (row.bin(value_of(mid)) >= b) hi = mid; else lo = mid + 1;
    }
    sh.range[threadIdx.x] = lo;
  }
  __syncthreads();
  uint32_t lo = sh.range[0], hi = sh.range[1];  // hi exclusive
  for (;;) {
    const uint32_t width = hi - lo;
    int shift = 0;
    while ((width - 1) >> shift >= (uint32_t)kBins) ++shift;
    for (int i = threadIdx.x; i < kBins; i += kThreads) sh.count[i] = sh.lo[i] = sh.hi[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const uint32_t k = key_of(vals[i]);
      if (k - lo < width) add_to_bin(sh, (int)((k - lo) >> shift), row.weight(vals[i]));
    }
    sum_bins(cluster, sh, 1, n, rank);
    find_bin(cluster, sh, 1, n, by_count, target - (by_count ? (u64)count_before : weight_before));
    weight_before += sh.found_weight_before;
    count_before += sh.found_count_before;
    const uint32_t first = lo + ((uint32_t)sh.found_bin << shift);
    if (shift == 0) {
      Cut cut;
      cut.key = first;
      const u64 each = row.weight(value_of(first));
      u64 ties = by_count ? target - count_before
                          : each > 0 ? (target - weight_before + each - 1) / each : 1;
      if (ties < 1) ties = 1;
      if (ties > sh.found_count) ties = sh.found_count;
      cut.ties = (uint32_t)ties;
      cut.weight = weight_before + ties * each;
      return cut;
    }
    lo = first;
    hi = min(hi, first + (1u << shift));
  }
}

template <typename T>
__device__ __forceinline__ float widen(T v);
template <>
__device__ __forceinline__ float widen<float>(float v) { return v; }
template <>
__device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

__device__ __forceinline__ float clean(float v) { return v != v ? -INFINITY : v + 0.0f; }

// Copies the slice to shared memory as floats; returns this thread's maximum.
template <typename T>
__device__ __forceinline__ float load_slice(const T* src, float* vals, int len) {
  float mx = -INFINITY;
  constexpr int kVec = 16 / sizeof(T);
  int done = 0;
  if ((reinterpret_cast<uintptr_t>(src) & 15u) == 0) {
    done = len / kVec * kVec;
    constexpr int kAhead = 4;
    for (int base = threadIdx.x * kVec; base < done; base += kAhead * kThreads * kVec) {
      uint4 r[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = base + k * kThreads * kVec;
        if (i < done) r[k] = __ldcs(reinterpret_cast<const uint4*>(src + i));
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = base + k * kThreads * kVec;
        if (i >= done) break;
        const uint32_t w[4] = {r[k].x, r[k].y, r[k].z, r[k].w};
        float f[kVec];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (sizeof(T) == 4) {
            f[j] = clean(__uint_as_float(w[j]));
          } else {
            f[2 * j] = clean(__uint_as_float(w[j] << 16));
            f[2 * j + 1] = clean(__uint_as_float(w[j] & 0xffff0000u));
          }
        }
#pragma unroll
        for (int j = 0; j < kVec; j += 4) {
          *reinterpret_cast<float4*>(vals + i + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
          mx = fmaxf(fmaxf(mx, fmaxf(f[j], f[j + 1])), fmaxf(f[j + 2], f[j + 3]));
        }
      }
    }
  }
  for (int i = done + threadIdx.x; i < len; i += kThreads) {
    const float v = clean(widen<T>(src[i]));
    vals[i] = v;
    mx = fmaxf(mx, v);
  }
  return mx;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_rows_cluster(const SampleParams p) {
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  float* vals = reinterpret_cast<float*>(smem + ((sizeof(Shared) + 15) & ~size_t(15)));
  const int n = (int)cluster_size(), rank = (int)cluster_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t i_row = blockIdx.x / n;
  if (threadIdx.x < 64) sh.table[threadIdx.x] = exp2(threadIdx.x / 64.0);
  for (int i = threadIdx.x; i < kBins; i += kThreads) sh.count[i] = sh.lo[i] = sh.hi[i] = 0;
  griddep_wait();
  griddep_launch_dependents();

  const int start = min(rank * p.slice, p.vocab), len = min(p.slice, p.vocab - start);
  float mx = load_slice<T>(static_cast<const T*>(p.logits) + i_row * p.ld + start, vals, len);
  mx = warp_max(mx);
  if (lane == 0) sh.warp_max[warp] = mx;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWarps; ++w) mx = fmaxf(mx, sh.warp_max[w]);
    sh.row_max = mx;
  }
  cluster.sync();
  Row row;
  row.table = sh.table;
  row.max = -INFINITY;
  for (int r = 0; r < n; ++r) row.max = fmaxf(row.max, cluster.map_shared_rank(&sh, r)->row_max);

  float temperature = p.temperature ? __ldg(p.temperature + i_row) : 1.f;
  int top_k = p.top_k ? __ldg(p.top_k + i_row) : 0;
  const float top_p = p.top_p ? __ldg(p.top_p + i_row) : 1.f;
  const float min_p = p.min_p ? __ldg(p.min_p + i_row) : 0.f;
  if (!(temperature > 0.f)) { temperature = 1.f; top_k = 1; }
  row.inv_t = 1.0 / (double)temperature;
  row.bin_scale = (float)((double)kBinsPerUnit * row.inv_t);

  // everything below is uniform over the cluster: the same row, the same parameters, the same sums
  Cut cut;
  cut.key = 0xffffffffu;  // nothing cut off
  cut.ties = 0;
  if (row.max > -INFINITY) {
    if (top_k == 1) {
      cut.key = key_of(row.max);
      cut.ties = 1;
    } else if ((top_k > 1 && top_k < p.vocab) || top_p < 1.f) {
      for (int i = threadIdx.x; i < len; i += kThreads) {
        const float v = vals[i];
        const int b = row.bin(v);
        if (b < kBins) add_to_bin(sh, b, row.weight(v));
      }
      sum_bins(cluster, sh, 0, n, rank);
      u64 total = 0;
      uint32_t eligible = 0;
      for (int r = 0; r < n; ++r) {
        const Shared* peer = cluster.map_shared_rank(&sh, r);
        total += peer->slice_weight[0];
        eligible += peer->slice_count[0];
      }
      if (top_k > 1 && (uint32_t)top_k < eligible) {
        cut = search(cluster, sh, row, vals, len, n, rank, true, (u64)top_k);
        total = cut.weight;
      }
      if (top_p < 1.f) {
        const double need = ceil((double)fmaxf(top_p, 0.f) * (double)total);
        cut = search(cluster, sh, row, vals, len, n, rank, false, need < 1.0 ? 1ull : (u64)need);
      }
    }
  }
  // (NaN and values below 0 filter nothing; a weight of zero units is never kept)
  const u64 min_weight = min_p > 0.f ? max((u64)ceil((double)fminf(min_p, 1.f) * (double)(1ull << kFixed)), 1ull) : 1ull;

  // Kept weight of this warp's contiguous share of the slice: what lies above the cut, and how many lie on it.
  const int share = ((len + kWarps - 1) / kWarps + 31) / 32 * 32;
  const int w_begin = min(warp * share, len), w_end = min(w_begin + share, len);
  u64 above = 0;
  uint32_t equal = 0;
  if (row.max > -INFINITY) {
    for (int i = w_begin + lane; i < w_end; i += 32) {
      const uint32_t k = key_of(vals[i]);
      if (k < cut.key) {
        const u64 w = row.weight(vals[i]);
        if (w >= min_weight) above += w;
      } else if (k == cut.key) {
        ++equal;
      }
    }
  }
  u64 each = cut.ties > 0 ? row.weight(value_of(cut.key)) : 0;  // weight of a logit on the cut
  if (each < min_weight) each = 0;
  above = warp_sum_u64(above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) { sh.warp_weight[warp] = above; sh.warp_count[warp] = equal; }
  __syncthreads();
  if (threadIdx.x == 0) {
    u64 a = 0;
    uint32_t e = 0;
    for (int w = 0; w < kWarps; ++w) { a += sh.warp_weight[w]; e += sh.warp_count[w]; }
    sh.above_weight = a;
    sh.equal_count = e;
  }
  cluster.sync();
  u64 total = 0, before = 0;
  uint32_t equal_total = 0, equal_before = 0;
  for (int r = 0; r < n; ++r) {
    const Shared* peer = cluster.map_shared_rank(&sh, r);
    if (r == rank) { before = total; equal_before = equal_total; }
    const uint32_t e = peer->equal_count;
    const uint32_t kept = equal_total >= cut.ties ? 0 : min(e, cut.ties - equal_total);
    total += peer->above_weight + kept * each;
    equal_total += e;
  }
  cluster.sync();  // nobody reads another CTA's memory from here on

  if (total == 0) {
    if (rank == 0 && threadIdx.x == 0) {
      p.tokens[i_row] = -1;
      if (p.probs) p.probs[i_row] = 0.f;
    }
    return;
  }
  float u = __ldg(p.u + i_row);
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;  // NaN: 0
  const u64 target = __umul64hi(total, (u64)((double)u * 18446744073709551616.0));  // floor(u * total) < total
  for (int w = 0; w < warp; ++w) {
    const uint32_t kept = equal_before >= cut.ties ? 0 : min(sh.warp_count[w], cut.ties - equal_before);
    before += sh.warp_weight[w] + kept * each;
    equal_before += sh.warp_count[w];
  }
  const uint32_t own_kept = equal_before >= cut.ties ? 0 : min(equal, cut.ties - equal_before);
  if (target < before || target >= before + above + own_kept * each) return;
  // this warp's share holds the token: walk it in index order
  for (int base = w_begin; base < w_end; base += 32) {
    const int i = base + lane;
    u64 w = 0;
    uint32_t k = 0xffffffffu;
    if (i < w_end) k = key_of(vals[i]);
    const unsigned on_cut = __ballot_sync(0xffffffffu, i < w_end && k == cut.key);
    if (i < w_end) {
      if (k < cut.key) {
        w = row.weight(vals[i]);
        if (w < min_weight) w = 0;
      } else if (k == cut.key && equal_before + __popc(on_cut & ((1u << lane) - 1u)) < cut.ties) {
        w = each;
      }
    }
    equal_before += __popc(on_cut);
    const u64 upto = before + warp_scan_u64(w);
    const unsigned past = __ballot_sync(0xffffffffu, upto > target);
    if (past) {
      if (lane == __ffs(past) - 1) {
        p.tokens[i_row] = start + i;
        if (p.probs) p.probs[i_row] = (float)((double)w / (double)total);
      }
      return;
    }
    before = __shfl_sync(0xffffffffu, upto, 31);
  }
}

// Slices of at most 16384 logits (64 KiB: two CTAs to an SM) where 8 CTAs allow it, and as many CTAs per row as it takes
// to give every SM some when rows are few.
int cluster_for(int64_t rows, int64_t vocab) {
  int n = 1;
  while (n < kMaxCluster && (vocab > 16384 * (int64_t)n || (rows * n < sm_count() && vocab > 2048 * (int64_t)n))) n *= 2;
  return n;
}

template <typename T>
pd_status launch(const SampleParams& p, int64_t rows, cudaStream_t s) {
  const int n = cluster_for(rows, p.vocab);
  SampleParams q = p;
  q.slice = (int)(((p.vocab + n - 1) / n + 7) / 8 * 8);
  const size_t fixed = (sizeof(Shared) + 15) & ~size_t(15);
  constexpr int kMaxSmem = (int)((sizeof(Shared) + 15) / 16 * 16) + (int)(kMaxVocab / kMaxCluster) * 4;
  static_assert(kMaxSmem <= 227 * 1024, "the longest slice fits");
  static PerDeviceFlag smem_allowed;
  if (pd_status st = allow_dynamic_smem(sample_rows_cluster<T>, kMaxSmem, smem_allowed); st != PD_OK) return st;
  logf("sample %lld x %d: clusters of %d CTAs", (long long)rows, p.vocab, n);
  launch_pdl_cluster(sample_rows_cluster<T>, dim3((unsigned)(rows * n)), dim3(kThreads), (unsigned)n,
                     fixed + (size_t)q.slice * 4, s, q);
  return check_launch();
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_sample(const void* logits, pd_dtype dtype, int64_t rows, int64_t vocab, int64_t ld,
                               const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                               const float* u, int32_t* tokens, float* probs, cudaStream_t stream) {
  if (rows < 0 || vocab <= 0 || ld < vocab || (dtype != PD_BF16 && dtype != PD_F32)) return PD_ERR_BAD_SHAPE;
  if (vocab > pd::kMaxVocab || rows > 0x7fffffff / pd::kMaxCluster) return PD_ERR_UNSUPPORTED;
  if (rows == 0) return PD_OK;
  if (!logits || !u || !tokens) return PD_ERR_NULL_POINTER;
  auto bits = [](const void* q) { return reinterpret_cast<uintptr_t>(q); };
  if ((bits(logits) & (dtype == PD_F32 ? 3u : 1u)) ||
      ((bits(temperature) | bits(top_k) | bits(top_p) | bits(min_p) | bits(u) | bits(tokens) | bits(probs)) & 3u))
    return PD_ERR_ALIGNMENT;
  if (pd_status st = pd::require_sm100(); st != PD_OK) return st;
  pd::SampleParams p{logits, temperature, top_p, min_p, u, top_k, tokens, probs, ld, (int)vocab, 0};
  return dtype == PD_F32 ? pd::launch<float>(p, rows, stream) : pd::launch<__nv_bfloat16>(p, rows, stream);
}
