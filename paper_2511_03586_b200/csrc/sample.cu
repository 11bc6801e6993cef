// One token per row of logits under temperature, top-k, top-p and min-p, from a given random number:
//
//   w[j] = exp((logits[j] - max) / T), ranked by logit, then by index; keep the first top_k, of these the shortest
//   leading run that reaches top_p of their weight, of these the ones with w >= min_p; draw the first index at which
//   the running kept weight exceeds u times its total.
//
// The row is never sorted as a whole.  A cut is "the first rank at which a running sum reaches a target", and a histogram
// over value (bins of 1/64 in (max - logit) / T) says which bin holds it; the logits of that bin, a few hundred of a
// hundred thousand, are gathered and sorted by (value, index), and the cut is the last kept one of them.
//   top-k            : histogram of counts; everything down to the bin of rank k is gathered, and the rest (top-p, min-p,
//                      the draw) happens on that short list.
//   top-p, no top-k  : the total weight exactly; then a histogram of approximate weights (one 32-bit atomic per logit in
//                      units of 2^-31 of the total, none for logits that are too light to come before the cut), whose
//                      error is bounded, so that one or two bins surely hold the cut; then the exact weight above them.
//   neither          : exact sums alone.
// The token is then found by prefix sums over warps' shares, and by a scan of one warp's share.
// Rows whose candidates do not fit the list (thousands of equal logits, a very large k) take histograms of exact weights
// over ever finer ranges of values instead, until a bin is a single value.
//
// Weights are summed as integers in units of 2^-44 of the largest weight (a row of 327680 weights stays below 2^63).
// Integer sums do not depend on their order, so atomics and any split over threads give the same bits, and the border of
// a cut, which decides between two tokens, is where the 64-bit definition has it: the exponential is evaluated in double
// precision (2^(n/512) from a table, the rest by its Taylor series to the third power: (ln 2 / 1024)^4 / 4! = 9e-15, a
// sixth of a unit).
//
// HBM-bound in principle: the logits are read once, 4 (or 2) bytes each, and held in the shared memory of a cluster of
// 1 to 8 CTAs (distributed by contiguous slices, so that index order is slice order).  In fact the passes over shared
// memory, the double-precision exponentials (ten operations each) and the cluster's barriers weigh more.
#include <cooperative_groups.h>

#include <cmath>

#include "pd_common.cuh"

namespace pd {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;           // bins of 1/64 in z = (max - logit) / T, up to z = 32 (weight 2^-46: zero units)
constexpr float kBinsPerUnit = 64.f;
constexpr int kList = 2048;           // candidates that are sorted
constexpr int kSlowBins = 1024;       // bins of a step of the search without a list
constexpr int kTable = 512;
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

// A float (not subnormal) as a double, by its bits: conversion instructions run at a quarter of the rate of additions.
__device__ __forceinline__ double as_double(float v) {
  const uint32_t b = __float_as_uint(v);
  const uint32_t hi = (b & 0x80000000u) | (((b & 0x7fffffffu) >> 3) + 0x38000000u);
  return (b << 1) != 0 ? __hiloint2double((int)hi, (int)(b << 29)) : 0.0;
}

struct Row {
  float max;
  double max_d;
  double per_step;   // kTable / (T ln 2): (logit - max) in 512ths of a factor of two
  float bin_scale;   // kBinsPerUnit / T
  float exp_scale;   // log2(e) / T
  const double* table;
  // weight of logit v in units of 2^-44
  __device__ __forceinline__ u64 weight(float v) const {
    if (v == max) return 1ull << kFixed;
    constexpr double kLn2 = 0.69314718055994530942;
    constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits hold the rounded integer
    const double y = (as_double(v) - max_d) * per_step;
    if (!(y > -32.0 / kLn2 * kTable) || v == -INFINITY) return 0;
    const double r = y + kMagic;
    const int n = (int)__double2loint(r);
    constexpr double c = kLn2 / kTable;
    const double f = y - (r - kMagic);
    double q = fma(c * c * c / 6.0, f, c * c / 2.0);
    q = fma(q, f, c);
    q = fma(q, f, 1.0);
    q *= table[n & (kTable - 1)];  // in [0.99, 2)
    q = __hiloint2double(__double2hiint(q) + (((n >> 9) + kFixed) << 20), __double2loint(q));  // times 2^(n / 512 + 44)
    const double whole = q + 4503599627370496.0;  // 2^52: rounds to an integer
    return (u64)__double_as_longlong(whole) & ((1ull << 52) - 1);
  }
  // bin: a monotone function of v (each rounding is monotone); kBins for weights of zero
  __device__ __forceinline__ int bin(float v) const {
    if (v == max) return 0;
    const float t = (max - v) * bin_scale;
    return t < (float)kBins ? (int)t : kBins;
  }
  // approximate weight relative to the largest: the exponent is at most 47, so its rounding (two steps of 2^-24) is below
  // 47 * 2^-23 = 6e-6, and the exponential's own error 2^-22; together below 1e-5 of the weight
  __device__ __forceinline__ float approx(float v) const {
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v == max ? 0.f : (v - max) * exp_scale));
    return e;
  }
};
static_assert(kTable == 512 && kTable == kThreads, "weight() shifts by 9, and every thread fills an entry");
constexpr double kApproxError = 2e-5;  // twice approx()'s bound

struct SlowSearch {
  // own histogram (weights in two halves), then the cluster's sums of the bins this CTA owns (first level, later levels)
  uint32_t count[kSlowBins], lo[kSlowBins], hi[kSlowBins];
  uint32_t sum_count[2][kSlowBins];
  u64 sum_weight[2][kSlowBins];
};
struct FastSearch {
  uint32_t hist[kBins];  // own histogram
  uint32_t sum[kBins];   // the cluster's
  u64 list[kList];       // candidates as (key, index), in CTA 0
};

struct Shared {
  double table[kTable];
  union {
    SlowSearch slow;
    FastSearch fast;
  };
  // filled by the cluster's CTAs, entry r by CTA r (peer_max and peer_weight in every CTA, the rest in CTA 0 alone)
  float peer_max[kMaxCluster];
  u64 peer_weight[kMaxCluster];
  uint32_t peer_candidates[kMaxCluster];
  u64 share_weight[kMaxCluster * kWarps];  // kept weight of every warp's share, candidates not included at first
  uint32_t candidates;
  uint32_t first_max;
  // search without a list: published to the cluster
  u64 slice_weight[2];
  uint32_t slice_count[2];
  u64 above_weight;
  uint32_t equal_count;
  // scratch of one CTA
  u64 warp_weight[kWarps];
  uint32_t warp_count[kWarps];
  float warp_max[kWarps];
  // result of a search step
  int found_bin, found_bin2;
  u64 found_weight_before, found_weight;
  uint32_t found_count_before, found_count;
  uint32_t range[2];
  uint32_t token;
  u64 token_weight, total;
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
  atomicAdd(&sh.slow.count[b], 1u);
  const uint32_t lo = (uint32_t)w;
  const uint32_t before = atomicAdd(&sh.slow.lo[b], lo);
  const uint32_t hi = (uint32_t)(w >> 32) + (before + lo < before ? 1u : 0u);
  if (hi) atomicAdd(&sh.slow.hi[b], hi);
}

// Sums the cluster's histograms: CTA r gets the bins [r, r + 1) * kSlowBins / n, and every CTA the sums over these slices of
// bins.  `level` 0 keeps the sums of the first histogram for a second search.
__device__ void sum_bins(cg::cluster_group& cluster, Shared& sh, int level, int n, int rank) {
  cluster.sync();  // every histogram is complete
  const int own = kSlowBins / n;
  u64 tw = 0;
  uint32_t tc = 0;
  for (int i = threadIdx.x; i < own; i += kThreads) {
    const int b = rank * own + i;
    u64 w = 0;
    uint32_t c = 0;
    for (int r = 0; r < n; ++r) {
      const Shared* peer = cluster.map_shared_rank(&sh, r);
      c += peer->slow.count[b];
      w += ((u64)peer->slow.hi[b] << 32) + peer->slow.lo[b];
    }
    sh.slow.sum_count[level][i] = c;
    sh.slow.sum_weight[level][i] = w;
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
  const int own = kSlowBins / n;
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
  u64 w[kSlowBins / kThreads], tw = 0;
  uint32_t c[kSlowBins / kThreads], tc = 0;
#pragma unroll
  for (int j = 0; j < kSlowBins / kThreads; ++j) {
    const int i = threadIdx.x * per + j;
    const bool in = j < per && i < own;
    w[j] = in ? peer->slow.sum_weight[level][i] : 0;
    c[j] = in ? peer->slow.sum_count[level][i] : 0;
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
  for (int j = 0; j < kSlowBins / kThreads; ++j) {
    if (c[j] > 0 && (by_count ? (u64)rc : rw) < target) atomicMax(&sh.found_bin, (int)threadIdx.x * per + j);
    rw += w[j];
    rc += c[j];
  }
  __syncthreads();
  rw = w0 + sw - tw;
  rc = c0 + sc - tc;
#pragma unroll
  for (int j = 0; j < kSlowBins / kThreads; ++j) {
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

// The cut of the search without a list: logits with a smaller key are kept, of those with this key the first `ties` by index.
struct SlowCut {
  uint32_t key;
  uint32_t ties;
  u64 weight;  // of everything kept
};

// First level already in sh.sum_*[0]: descends to the single logit value at which the running count or weight reaches
// `target`.
__device__ SlowCut search(cg::cluster_group& cluster, Shared& sh, const Row& row, const float* vals, int len, int n, int rank,
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
      if (row.bin(value_of(mid)) / 2 >= b) hi = mid; else lo = mid + 1;
    }
    sh.range[threadIdx.x] = lo;
  }
  __syncthreads();
  uint32_t lo = sh.range[0], hi = sh.range[1];  // hi exclusive
  for (;;) {
    const uint32_t width = hi - lo;
    int shift = 0;
    while ((width - 1) >> shift >= (uint32_t)kSlowBins) ++shift;
    for (int i = threadIdx.x; i < kSlowBins; i += kThreads) sh.slow.count[i] = sh.slow.lo[i] = sh.slow.hi[i] = 0;
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
      SlowCut cut;
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

// NaN counts as -inf, -0 and subnormal logits as +0.
__device__ __forceinline__ float clean(float v) {
  if (v != v) return -INFINITY;
  return fabsf(v) < 1.17549435e-38f ? 0.f : v;
}

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

// ---- one CTA's helpers ---------------------------------------------------------------
// Inclusive scan of one value per thread over the CTA.
__device__ __forceinline__ u64 block_scan_u64(Shared& sh, u64 v) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __syncthreads();
  v = warp_scan_u64(v);
  if (lane == 31) sh.warp_weight[warp] = v;
  __syncthreads();
  for (int k = 0; k < warp; ++k) v += sh.warp_weight[k];
  return v;
}

// Sorts list[0 ... size) ascending; size a power of two.
__device__ void sort_list(u64* list, int size) {
  for (int run = 2; run <= size; run <<= 1)
    for (int step = run >> 1; step > 0; step >>= 1) {
      for (int i = threadIdx.x; i < size / 2; i += kThreads) {
        const int a = 2 * i - (i & (step - 1)), b = a + step;
        const u64 x = list[a], y = list[b];
        if ((x > y) == ((a & run) == 0)) { list[a] = y; list[b] = x; }
      }
      __syncthreads();
    }
}

// Writes a row's result.
__device__ __forceinline__ void write_token(const SampleParams& p, int64_t row, uint32_t token, u64 weight, u64 total) {
  p.tokens[row] = (int32_t)token;
  if (p.probs) p.probs[row] = (float)((double)weight / (double)total);
}

__device__ __forceinline__ u64 draw_target(const SampleParams& p, int64_t row, u64 total) {
  float u = __ldg(p.u + row);
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;                                    // NaN: 0
  return __umul64hi(total, (u64)((double)u * 18446744073709551616.0));            // floor(u * total) < total
}

// Sums the cluster's histograms into every CTA's fast.sum: CTA r adds up bins [r, r + 1) * kBins / n and hands them out.
__device__ void sum_histograms(cg::cluster_group& cluster, Shared& sh, int n, int rank) {
  cluster.sync();  // every histogram is complete
  const int own = kBins / n;
  for (int i = threadIdx.x; i < own; i += kThreads) {
    const int b = rank * own + i;
    uint32_t part[kMaxCluster], c = 0;
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) part[r] = r < n ? cluster.map_shared_rank(&sh, r)->fast.hist[b] : 0;
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) c += part[r];
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r)
      if (r < n) cluster.map_shared_rank(&sh, r)->fast.sum[b] = c;
  }
  cluster.sync();  // the sums are in, and nobody reads a histogram any more
}

// sh.found_bin, found_bin2: the first bins whose running sum reaches t1 and t2 (kBins - 1 if none does);
// found_count: the running sum through found_bin2.
__device__ void locate(Shared& sh, u64 t1, u64 t2) {
  constexpr int kPer = kBins / kThreads;
  uint32_t c[kPer];
  u64 sum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) { c[j] = sh.fast.sum[threadIdx.x * kPer + j]; sum += c[j]; }
  const u64 upto = block_scan_u64(sh, sum);
  if (threadIdx.x == kThreads - 1) {
    sh.found_bin = sh.found_bin2 = kBins - 1;
    sh.found_count = (uint32_t)upto;
  }
  __syncthreads();
  u64 run = upto - sum;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const u64 before = run;
    run += c[j];
    if (before < t1 && run >= t1) sh.found_bin = threadIdx.x * kPer + j;
    if (before < t2 && run >= t2) { sh.found_bin2 = threadIdx.x * kPer + j; sh.found_count = (uint32_t)run; }
  }
  __syncthreads();
}

// CTA 0: sorts its n candidates by (key, index) in place and pads them to a power of two.
__device__ void sort_candidates(Shared& sh, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += kThreads) sh.fast.list[i] = ~0ull;
  __syncthreads();
  sort_list(sh.fast.list, size);
}

__device__ __forceinline__ u64 candidate(float v, int index) { return (u64)key_of(v) << 32 | (uint32_t)index; }
__device__ __forceinline__ float candidate_value(u64 c) { return value_of((uint32_t)(c >> 32)); }

// Hands a candidate to CTA 0.
__device__ __forceinline__ void add_candidate(Shared* first, float v, int index) {
  const uint32_t at = atomicAdd(&first->candidates, 1u);
  if (at < (uint32_t)kList) first->fast.list[at] = candidate(v, index);
}

// CTA 0, after top-k: the first `k` of the n sorted candidates are what is left of the row; top-p, min-p and the draw.
__device__ void finish_list(const SampleParams& p, Shared& sh, const Row& row, int64_t i_row, int n, int k, float top_p,
                            u64 min_weight) {
  constexpr int kPer = kList / kThreads;
  sort_candidates(sh, n);
  n = min(n, k);
  u64* list = sh.fast.list;
  // the kept run: ranks whose predecessors weigh less than top_p of all; then min-p
  u64 w[kPer], sum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = threadIdx.x * kPer + j;
    w[j] = i < n ? row.weight(candidate_value(list[i])) : 0;
    sum += w[j];
  }
  u64 upto = block_scan_u64(sh, sum);
  if (threadIdx.x == kThreads - 1) sh.total = upto;
  __syncthreads();
  u64 need = ~0ull;
  if (top_p < 1.f) need = max((u64)ceil((double)fmaxf(top_p, 0.f) * (double)sh.total), 1ull);
  u64 before = upto - sum;
  // what is kept goes on as (index, rank), the rest is pushed to the end
  u64 entry[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = threadIdx.x * kPer + j;
    const bool kept = i < n && before < need && w[j] >= min_weight;
    entry[j] = kept ? (list[i] << 32) | (list[i] >> 32) : ~0ull;  // (index, key)
    before += w[j];
  }
  __syncthreads();
  int size = 2;
  while (size < n) size <<= 1;
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if ((int)threadIdx.x * kPer + j < size) list[threadIdx.x * kPer + j] = entry[j];
  __syncthreads();
  sort_list(list, size);
  sum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = threadIdx.x * kPer + j;
    entry[j] = i < size ? list[i] : ~0ull;
    w[j] = entry[j] != ~0ull ? row.weight(value_of((uint32_t)entry[j])) : 0;
    sum += w[j];
  }
  upto = block_scan_u64(sh, sum);
  if (threadIdx.x == kThreads - 1) sh.total = upto;
  __syncthreads();
  const u64 target = draw_target(p, i_row, sh.total);
  before = upto - sum;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    if (before <= target && target < before + w[j]) write_token(p, i_row, (uint32_t)(entry[j] >> 32), w[j], sh.total);
    before += w[j];
  }
}

// CTA 0, top-p without top-k or no cut at all: share_weight holds the kept weight of every warp's share up to the
// candidates, `last` the last kept (key, index), ~0 for no cut.  Finds the share that the draw falls into and scans it
// (its logits are read again from global memory: the other CTAs are gone).
template <typename T>
__device__ void finish_shares(const SampleParams& p, Shared& sh, const Row& row, int64_t i_row, int n, int share, u64 last,
                              u64 min_weight) {
  __syncthreads();
  const u64 mine = threadIdx.x < n * kWarps ? sh.share_weight[threadIdx.x] : 0;
  const u64 upto = block_scan_u64(sh, mine);
  if (threadIdx.x == kThreads - 1) sh.total = upto;
  __syncthreads();
  const u64 total = sh.total;
  const u64 target = draw_target(p, i_row, total);
  if (upto - mine <= target && target < upto) {
    sh.token = threadIdx.x;
    sh.found_weight_before = upto - mine;
  }
  __syncthreads();
  const int cta = sh.token / kWarps, warp = sh.token % kWarps;
  const int start = cta * p.slice + warp * share;
  const int end = min(min(start + share, (cta + 1) * p.slice), p.vocab);
  u64 before = sh.found_weight_before;
  const T* src = static_cast<const T*>(p.logits) + i_row * p.ld;
  for (int base = start; base < end; base += kThreads) {  // (one step for shares of up to 512)
    const int i = base + threadIdx.x;
    u64 w = 0;
    if (i < end) {
      const float v = clean(widen<T>(src[i]));
      if (candidate(v, i) <= last) w = row.weight(v);
      if (w < min_weight) w = 0;
    }
    const u64 to = before + block_scan_u64(sh, w);
    if (to - w <= target && target < to) write_token(p, i_row, i, w, total);
    if (threadIdx.x == kThreads - 1) sh.token_weight = to;
    __syncthreads();
    before = sh.token_weight;
  }
}

template <typename T>
__device__ void slow_path(cg::cluster_group& cluster, const SampleParams& p, Shared& sh, const Row& row, const float* vals,
                          int64_t i_row, int start, int len, int n, int rank, int top_k, float top_p, u64 min_weight) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  SlowCut cut;
  cut.key = 0xffffffffu;  // nothing cut off
  cut.ties = 0;
  cluster.sync();  // the list's memory is free
  for (int i = threadIdx.x; i < kSlowBins; i += kThreads) sh.slow.count[i] = sh.slow.lo[i] = sh.slow.hi[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < len; i += kThreads) {
    const float v = vals[i];
    const int b = row.bin(v) / 2;
    if (b < kSlowBins) add_to_bin(sh, b, row.weight(v));
  }
  sum_bins(cluster, sh, 0, n, rank);
  u64 kept_total = 0;
  uint32_t eligible = 0;
  for (int r = 0; r < n; ++r) {
    const Shared* peer = cluster.map_shared_rank(&sh, r);
    kept_total += peer->slice_weight[0];
    eligible += peer->slice_count[0];
  }
  if (top_k > 1 && (uint32_t)top_k < eligible) {
    cut = search(cluster, sh, row, vals, len, n, rank, true, (u64)top_k);
    kept_total = cut.weight;
  }
  if (top_p < 1.f) {
    const double need = ceil((double)fmaxf(top_p, 0.f) * (double)kept_total);
    cut = search(cluster, sh, row, vals, len, n, rank, false, need < 1.0 ? 1ull : (u64)need);
  }

  // Kept weight of this warp's contiguous share of the slice: what lies above the cut, and how many lie on it.
  const int share = ((len + kWarps - 1) / kWarps + 31) / 32 * 32;
  const int w_begin = min(warp * share, len), w_end = min(w_begin + share, len);
  u64 above = 0;
  uint32_t equal = 0;
  {
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

// Two CTAs to an SM: one's passes run while the other waits for its cluster.
template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_rows_cluster(const SampleParams p) {
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  float* vals = reinterpret_cast<float*>(smem + ((sizeof(Shared) + 15) & ~size_t(15)));
  const int n = (int)cluster_size(), rank = (int)cluster_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t i_row = blockIdx.x / n;
  sh.table[threadIdx.x] = exp2(threadIdx.x / (double)kTable);
  for (int i = threadIdx.x; i < kBins; i += kThreads) sh.fast.hist[i] = 0;
  if (threadIdx.x == 0) { sh.candidates = 0; sh.first_max = 0xffffffffu; }
  griddep_wait();
  griddep_launch_dependents();

  float temperature = p.temperature ? __ldg(p.temperature + i_row) : 1.f;
  int top_k = p.top_k ? __ldg(p.top_k + i_row) : 0;
  const float top_p = p.top_p ? __ldg(p.top_p + i_row) : 1.f;
  const float min_p = p.min_p ? __ldg(p.min_p + i_row) : 0.f;
  if (!(temperature > 0.f)) { temperature = 1.f; top_k = 1; }
  // (NaN and values below 0 filter nothing; a weight of zero units is never kept)
  const u64 min_weight = min_p > 0.f ? max((u64)ceil((double)fminf(min_p, 1.f) * (double)(1ull << kFixed)), 1ull) : 1ull;

  const int start = min(rank * p.slice, p.vocab), len = min(p.slice, p.vocab - start);
  float mx = load_slice<T>(static_cast<const T*>(p.logits) + i_row * p.ld + start, vals, len);
  mx = warp_max(mx);
  if (lane == 0) sh.warp_max[warp] = mx;
  __syncthreads();
  if (threadIdx.x < n) {
    for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, sh.warp_max[w]);
    cluster.map_shared_rank(&sh, threadIdx.x)->peer_max[rank] = mx;
  }
  cluster.sync();
  Row row;
  row.table = sh.table;
  row.max = -INFINITY;
  for (int r = 0; r < n; ++r) row.max = fmaxf(row.max, sh.peer_max[r]);
  const double inv_t = 1.0 / (double)temperature;
  row.max_d = row.max == INFINITY ? 0.0 : as_double(row.max);
  row.per_step = inv_t * (kTable / 0.69314718055994530942);
  row.bin_scale = (float)((double)kBinsPerUnit * inv_t);
  row.exp_scale = (float)(inv_t * 1.4426950408889634);
  if (row.max == INFINITY) {  // everything else weighs nothing
    row.max_d = 1e39;
    row.per_step = 1e300;
  }
  Shared* first = cluster.map_shared_rank(&sh, 0);

  // everything below is uniform over the cluster: the same row, the same parameters, the same sums
  if (row.max == -INFINITY) {
    if (rank == 0 && threadIdx.x == 0) {
      p.tokens[i_row] = -1;
      if (p.probs) p.probs[i_row] = 0.f;
    }
    return;
  }
  if (top_k == 1) {
    for (int i = threadIdx.x; i < len; i += kThreads)
      if (vals[i] == row.max) { atomicMin(&first->first_max, (uint32_t)(start + i)); break; }
    cluster.sync();
    if (rank == 0 && threadIdx.x == 0) write_token(p, i_row, sh.first_max, 1, 1);
    return;
  }
  const int share = ((p.slice + kWarps - 1) / kWarps + 31) / 32 * 32;  // of a warp, contiguous
  const int w_begin = min(warp * share, len), w_end = min(w_begin + share, len);
  if (top_k > 1 && top_k < p.vocab) {
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const int b = row.bin(vals[i]);
      if (b < kBins) atomicAdd(&sh.fast.hist[b], 1u);
    }
    sum_histograms(cluster, sh, n, rank);
    locate(sh, 1, (u64)top_k);
    const int bin = sh.found_bin2;
    const uint32_t count = sh.found_count;
    if (count > (uint32_t)kList) {
      slow_path<T>(cluster, p, sh, row, vals, i_row, start, len, n, rank, top_k, top_p, min_weight);
      return;
    }
    for (int i = threadIdx.x; i < len; i += kThreads)
      if (row.bin(vals[i]) <= bin) add_candidate(first, vals[i], start + i);
    cluster.sync();
    if (rank == 0) finish_list(p, sh, row, i_row, (int)count, top_k, top_p, min_weight);
    return;
  }
  if (top_p < 1.f) {
    u64 sum = 0;
    for (int i = threadIdx.x; i < len; i += kThreads) sum += row.weight(vals[i]);
    sum = warp_sum_u64(sum);
    if (lane == 0) sh.warp_weight[warp] = sum;
    __syncthreads();
    if (threadIdx.x < n) {
      sum = 0;
      for (int w = 0; w < kWarps; ++w) sum += sh.warp_weight[w];
      cluster.map_shared_rank(&sh, threadIdx.x)->peer_weight[rank] = sum;
    }
    cluster.sync();
    u64 total = 0;
    for (int r = 0; r < n; ++r) total += sh.peer_weight[r];
    const u64 need = max((u64)ceil((double)fmaxf(top_p, 0.f) * (double)total), 1ull);
    // Units of 2^-31 of the total.  The logits lighter than `light` weigh less than the tail behind the cut, all together.
    const double total_rel = (double)total / (double)(1ull << kFixed);  // in weights of the largest
    const float unit = (float)(2147483648.0 / total_rel);
    const float light = (float)(0.5 * (1.0 - (double)need / (double)total) * total_rel / p.vocab);
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const float v = vals[i], e = row.approx(v);
      const int b = row.bin(v);
      if (b < kBins && e >= light) atomicAdd(&sh.fast.hist[b], (uint32_t)(e * unit));
    }
    sum_histograms(cluster, sh, n, rank);
    // every weight is off by less than a unit and kApproxError of itself
    const u64 slack = (u64)p.vocab + (u64)(2147483648.0 * kApproxError);
    const u64 need_units = (u64)((double)need / (double)total * 2147483648.0);
    locate(sh, need_units > slack ? need_units - slack : 1, need_units + slack);
    // (the cut lies above `light` in any case)
    const int low = need_units > slack ? sh.found_bin : 0;
    const int high = min(sh.found_bin2, light > 0.f ? (int)(kBinsPerUnit * (1.f - ::logf(light))) : kBins - 1);
    u64 above = 0, kept = 0;
    uint32_t mine = 0;
    for (int i = w_begin + lane; i < w_end; i += 32) {
      const float v = vals[i];
      const int b = row.bin(v);
      if (b < low) {
        const u64 w = row.weight(v);
        above += w;
        if (w >= min_weight) kept += w;
      } else if (b <= high) {
        add_candidate(first, v, start + i);
        ++mine;
      }
    }
    above = warp_sum_u64(above);
    kept = warp_sum_u64(kept);
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) {
      first->share_weight[rank * kWarps + warp] = kept;
      sh.warp_weight[warp] = above;
      sh.warp_count[warp] = mine;
    }
    __syncthreads();
    if (threadIdx.x < n) {
      above = 0;
      mine = 0;
      for (int w = 0; w < kWarps; ++w) { above += sh.warp_weight[w]; mine += sh.warp_count[w]; }
      Shared* peer = cluster.map_shared_rank(&sh, threadIdx.x);
      peer->peer_weight[rank] = above;
      peer->peer_candidates[rank] = mine;
    }
    cluster.sync();
    uint32_t count = 0;
    u64 before = 0;
    for (int r = 0; r < n; ++r) { count += sh.peer_candidates[r]; before += sh.peer_weight[r]; }
    if (count > (uint32_t)kList) {
      slow_path<T>(cluster, p, sh, row, vals, i_row, start, len, n, rank, top_k, top_p, min_weight);
      return;
    }
    if (rank != 0) return;
    // the last candidate whose predecessors weigh less than `need`
    sort_candidates(sh, (int)count);
    constexpr int kPer = kList / kThreads;
    u64 w[kPer];
    sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      w[j] = i < (int)count ? row.weight(candidate_value(sh.fast.list[i])) : 0;
      sum += w[j];
    }
    if (threadIdx.x == 0) sh.token = 0;
    before += block_scan_u64(sh, sum) - sum;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = threadIdx.x * kPer + j;
      if (i < (int)count && before < need) {
        atomicMax(&sh.token, (uint32_t)i);
        if (w[j] >= min_weight) {
          const int index = (int)(uint32_t)sh.fast.list[i];
          const int cta = index / p.slice;
          atomicAdd(&sh.share_weight[cta * kWarps + (index - cta * p.slice) / share], w[j]);
        }
      }
      before += w[j];
    }
    __syncthreads();
    const u64 last = sh.fast.list[sh.token];
    finish_shares<T>(p, sh, row, i_row, n, share, last, min_weight);
    return;
  }
  u64 kept = 0;
  for (int i = w_begin + lane; i < w_end; i += 32) {
    const u64 w = row.weight(vals[i]);
    if (w >= min_weight) kept += w;
  }
  kept = warp_sum_u64(kept);
  if (lane == 0) first->share_weight[rank * kWarps + warp] = kept;
  cluster.sync();
  if (rank == 0) finish_shares<T>(p, sh, row, i_row, n, share, ~0ull, min_weight);
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
