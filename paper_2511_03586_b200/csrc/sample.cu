// One token per row of logits under temperature, top-k, top-p and min-p, from a given random number:
//
//   w[j] = exp((logits[j] - max) / T), ranked by logit, then by index; keep the first top_k, of these the shortest
//   leading run that reaches top_p of their weight, of these the ones with w >= min_p; draw the first index at which
//   the running kept weight exceeds u times its total.
//
// The row is never sorted as a whole.  A cut is "the first rank at which a running sum reaches a target", and a histogram
// of counts over value (bins of 1/64 in (max - logit) / T) says which bin holds it; the logits of that bin, a few hundred of
// a hundred thousand, are gathered in one CTA, where the search goes on over (value, index) until it is down to one.
//   top-k            : everything down to the bin of rank k is gathered, and the rest (top-p, min-p) happens on that list.
//   top-p, no top-k  : weights within a bin differ by 1.6 %, so the counts bound the weight before and behind every bin, and
//                      with these the bins, one to three of them, that can hold the cut; the exact weight of all, and of
//                      what lies above these bins, is then summed in one pass.
//   neither          : sums alone.
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
// memory, the double-precision exponentials (eight operations each) and the cluster's barriers weigh more: 256 x 128000
// fp32 logits with top-p take 180 us, 20 of which the bytes need; stopped after the maximum, 43; after the cut's bins are
// known, about 80; after the exact sums, 156 (the last three of a launch of 177).  CTAs of 256 threads and 128 registers take
// 202 us (against 184 then).  Two CTAs fit an SM up to vocabularies of about 145800; 151936 logits take 274 us.
#include <cooperative_groups.h>

#include <cmath>

#include "pd_common.cuh"

namespace pd {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;           // bins of 1/64 in z = (max - logit) / T, up to z = 32 (weight 2^-46: zero units)
constexpr float kBinsPerUnit = 64.f;
constexpr int kSlowBins = 1024;       // bins of a step of the search without a list
constexpr int kList = 2048;           // candidates that one CTA takes
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

// 2^(44 + i / 512), by the Taylor series of exp (22 terms: ln 2 to the 23rd over 23! is 1e-26).
struct PowerTable {
  double v[kTable];
  constexpr PowerTable() : v() {
    for (int i = 0; i < kTable; ++i) {
      const double x = 0.69314718055994530942 * i / kTable;
      double e = 1.0;
      for (int k = 22; k > 0; --k) e = 1.0 + e * x / k;
      v[i] = e * (double)(1ull << kFixed);
    }
  }
};
__device__ constexpr PowerTable kPowers{};

struct Row {
  float max;
  float floor;       // logits at or below it weigh nothing (half a unit is at z = -31.2): they are raised to it
  double max_d;
  double per_step;   // kTable / (T ln 2): (logit - max) in 512ths of a factor of two
  float bin_scale;   // kBinsPerUnit / T
  const double* table;  // 2^(44 + i / 512)

  __device__ void set(float row_max, float temperature) {
    max = row_max;
    max_d = (double)row_max;
    double t = (double)temperature;
    constexpr double kFloor = 33.0;
    floor = fminf(__double2float_rd(max_d - kFloor * t), value_of(key_of(row_max) + 1));  // at most the float below max
    // where T is far below the spacing of floats, everything but the largest weighs nothing anyway
    if (!(max_d - (double)floor <= 2.0 * kFloor * t)) t = (max_d - (double)floor) / kFloor;
    const double inv_t = 1.0 / t;
    per_step = inv_t * (kTable / 0.69314718055994530942);
    bin_scale = (float)((double)kBinsPerUnit * inv_t);
  }
  // 2^52 plus the weight of logit v in units of 2^-44: a whole number whose low bits are the weight.
  // Without branches, and with what the conversion, the double-precision and the integer pipe can each bear (integer
  // operations were the limit when the float was widened by its bits and the exceptions were selected at the end; now
  // the double-precision pipe, at half the rate of single precision, is: eight operations, each a step of the formula).
  __device__ __forceinline__ double biased_weight(float v) const {
    constexpr double kMagic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits hold the rounded integer
    const double d = (double)fmaxf(v, floor) - max_d;
    const double r = fma(d, per_step, kMagic);
    const int n = __double2loint(r);
    constexpr double c = 0.69314718055994530942 / kTable;
    const double f = fma(d, per_step, kMagic - r);
    double q = fma(c * c * c / 6.0, f, c * c / 2.0);
    q = fma(q, f, c);
    q = fma(q, f, 1.0);
    const double t = table[n & (kTable - 1)];
    const double t2 = __hiloint2double(__double2hiint(t) + ((n << 11) & 0xfff00000), __double2loint(t));  // times 2^(n >> 9)
    return fma(t2, q, kBias);  // rounds to an integer
  }
  static constexpr double kBias = 4503599627370496.0;  // 2^52
  static constexpr int kBiasHigh = 0x43300000;         // its upper word
  // the weight as an integer, and as a double (sums of up to 2^9 of them are exact)
  __device__ __forceinline__ u64 weight(float v) const {
    const double w = biased_weight(v);
    return (u64)(uint32_t)(__double2hiint(w) - kBiasHigh) << 32 | (uint32_t)__double2loint(w);
  }
  __device__ __forceinline__ double weight_d(float v) const { return biased_weight(v) - kBias; }
  // 2^23 plus the bin of v: a monotone function of v (each rounding is monotone), compared as a float, NaN (0 * inf) and
  // kBinEnd or more for weights of zero
  __device__ __forceinline__ float biased_bin(float v) const { return fmaf(max - v, bin_scale, kBinBias); }
  static constexpr float kBinBias = 8388608.f, kBinEnd = kBinBias + kBins;
  __device__ __forceinline__ int bin(float v) const {
    return __float_as_int(fminf(biased_bin(v), kBinEnd)) & 0xffff;  // (NaN: kBins)
  }
};
static_assert(kTable == 512 && kTable == kThreads, "weight() shifts by 9, and every thread fills an entry");

struct SlowSearch {
  // own histogram (weights in two halves), then the cluster's sums of the bins this CTA owns (first level, later levels)
  uint32_t count[kSlowBins], lo[kSlowBins], hi[kSlowBins];
  uint32_t sum_count[2][kSlowBins];
  u64 sum_weight[2][kSlowBins];
};
struct FastSearch {
  uint32_t hist[kBins / 2];  // own counts, two to a word (a slice has fewer than 2^16 logits)
  union {
    uint32_t sum[kBins];     // the cluster's
    u64 own[kList];          // then the CTA's candidates, then scratch of the search among all
  };
  u64 list[kList];           // candidates as (key, index), in CTA 0
};
static_assert(kMaxVocab / kMaxCluster < 65536);

struct Shared {
  double table[kTable];
  union {
    SlowSearch slow;
    FastSearch fast;
  };
  // filled by the cluster's CTAs, entry r by CTA r (the peer_ ones in every CTA, share_weight in CTA 0 alone)
  float peer_max[kMaxCluster];
  uint32_t peer_candidates[kMaxCluster];
  u64 peer_total[kMaxCluster], peer_above[kMaxCluster];
  u64 share_weight[kMaxCluster * kWarps];  // kept weight of every warp's share, candidates not included at first
  uint32_t candidates, own_candidates;
  uint32_t first_max;
  // search without a list: published to the cluster
  u64 slice_weight[2];
  uint32_t slice_count[2];
  u64 above_weight;
  uint32_t equal_count;
  // scratch of one CTA
  u64 warp_weight[kWarps];
  uint32_t warp_count[kWarps];
  u64 warp_high[kWarps];
  float2 warp_bounds[kWarps];
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

// NaN counts as -inf, -0 as +0.
__device__ __forceinline__ float clean(float v) { return fmaxf(v, -INFINITY) + 0.0f; }
// Two kinds of rows are mapped to ordinary ones, in shared memory, once their maximum is known.  With logits of +inf, these
// become 0 and all others -inf.  Where 33 T below the maximum is out of range, every finite logit is near -2^128:
// logits and T are scaled by a power of two.
enum class Remap { kNone, kInfinite, kScale };
constexpr float kRemapScale = 0x1p-64f;
__device__ __forceinline__ float remapped(float v, Remap how) {
  return how == Remap::kNone ? v : how == Remap::kScale ? v * kRemapScale : v == INFINITY ? 0.f : -INFINITY;
}

// Copies the slice to shared memory as floats; returns this thread's maximum.
template <typename T>
__device__ __forceinline__ float load_slice(const T* src, float* vals, int len) {
  float mx = -INFINITY;
  constexpr int kVec = 16 / sizeof(T);
  int done = 0;
  if ((reinterpret_cast<uintptr_t>(src) & 15u) == 0) {
    done = len / kVec * kVec;
    constexpr int kAhead = 8;
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
  if (threadIdx.x < 3 && len + threadIdx.x < (len + 3) / 4 * 4) vals[len + threadIdx.x] = -INFINITY;  // for_share's last group
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
#pragma unroll
  for (int k = 0; k < kWarps; ++k) v += k < warp ? sh.warp_weight[k] : 0;
  return v;
}

// f(v, i) for the logits of this warp's share: groups of four to a lane, the last group padded with -inf.
template <typename F>
__device__ __forceinline__ void for_share(const float* vals, int begin, int end, F&& f) {
#pragma unroll 2
  for (int i = begin + 4 * (int)(threadIdx.x & 31); i < end; i += 128) {
    const float4 v = *reinterpret_cast<const float4*>(vals + i);
    f(v.x, i);
    f(v.y, i + 1);
    f(v.z, i + 2);
    f(v.w, i + 3);
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

// Sums the cluster's histograms into every CTA's fast.sum.  The histograms stay as they are until the next cluster barrier.
constexpr int kEach = kBins / kThreads;
__device__ void sum_histograms(cg::cluster_group& cluster, Shared& sh, int n) {
  static_assert(kEach == 4, "a thread's bins are two words");
  cluster.sync();  // every histogram is complete
  uint2 part[kMaxCluster];
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r)
    part[r] = r < n ? reinterpret_cast<const uint2*>(cluster.map_shared_rank(&sh, r)->fast.hist)[threadIdx.x] : make_uint2(0, 0);
  uint4 sum = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) {
    sum.x += part[r].x & 0xffffu;
    sum.y += part[r].x >> 16;
    sum.z += part[r].y & 0xffffu;
    sum.w += part[r].y >> 16;
  }
  reinterpret_cast<uint4*>(sh.fast.sum)[threadIdx.x] = sum;
  __syncthreads();
}

// The first bin through which there are `rank` logits or more (the last bin if there are fewer in all): sh.found_bin, and
// their number, sh.found_count.
__device__ void locate_rank(Shared& sh, uint32_t rank) {
  uint32_t c[kEach], sum = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) { c[j] = sh.fast.sum[threadIdx.x * kEach + j]; sum += c[j]; }
  const uint32_t upto = (uint32_t)block_scan_u64(sh, sum);
  if (threadIdx.x == kThreads - 1) {
    sh.found_bin = kBins - 1;
    sh.found_count = upto;
  }
  __syncthreads();
  uint32_t run = upto - sum;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const uint32_t before = run;
    run += c[j];
    if (before < rank && run >= rank) {
      sh.found_bin = threadIdx.x * kEach + j;
      sh.found_count = run;
    }
  }
  __syncthreads();
}

// The bins that can hold the cut at the share `top_p` of all weight: the first bin b at which prefix(b) >= top_p (prefix(b) +
// suffix(b)), where prefix is the weight of the bins up to b and suffix that of the bins behind it, that is
//   (1 - top_p) prefix(b) >= top_p suffix(b).
// The logits of bin b lie within half a bin (and the rounding of bin()) of z = b / 64, so counts bound both sums from below
// and above: sh.found_bin is the first bin where the condition may hold, sh.found_bin2 the first where it must.
//
// Single precision will do: the sums are off by 2^-18 of themselves at most (40 additions and products of positive terms),
// and a term by what __expf is, 2 + 1.173 x steps at most, 39 or 5e-6 of itself at x = 32.  The terms' factors leave room for
// both: they are 8e-5 (lower) and 1.7e-4 (upper) away from the bounds they stand for.  Sums run from the far end, so that a
// small suffix, which a top_p near 1 is decided by, is not a difference of large numbers.
__device__ void locate_weight(Shared& sh, float top_p, int vocab) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float lo[kEach], hi[kEach], lo_sum = 0.f, hi_sum = 0.f;
  const int last = kBins - 1 - (int)threadIdx.x * kEach;  // this thread's bins: last, last - 1, ..
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const float c = (float)sh.fast.sum[last - j];                       // (below 2^24)
    const float mid = __expf(-(float)(last - j) / kBinsPerUnit);
    lo[j] = c * (mid * (1.f - 0.515f / kBinsPerUnit));                  // e^-x >= 1 - x, x = 0.51 / 64
    hi[j] = c * (mid * (1.f + 0.525f / kBinsPerUnit));                  // e^x <= 1 + x + x^2
    lo_sum += lo[j];
    hi_sum += hi[j];
  }
  float lo_upto = lo_sum, hi_upto = hi_sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float u = __shfl_up_sync(0xffffffffu, lo_upto, o), v = __shfl_up_sync(0xffffffffu, hi_upto, o);
    if (lane >= o) { lo_upto += u; hi_upto += v; }
  }
  float lo_run = __shfl_up_sync(0xffffffffu, lo_upto, 1), hi_run = __shfl_up_sync(0xffffffffu, hi_upto, 1);
  if (lane == 0) lo_run = hi_run = 0.f;
  if (lane == 31) sh.warp_bounds[warp] = make_float2(lo_upto, hi_upto);
  if (threadIdx.x == 0) sh.found_bin = sh.found_bin2 = kBins - 1;
  __syncthreads();
  float lo_all = 0.f, hi_all = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const float2 b = sh.warp_bounds[w];
    if (w == warp) { lo_run += lo_all; hi_run += hi_all; }  // now the weight behind this thread's bins
    lo_all += b.x;
    hi_all += b.y;
  }
  // Weights are rounded to units, half a unit each; the differences below are off by 2^-18 of the sum of all.
  const float units = vocab * (1.f / (float)(1ull << kFixed)), off = hi_all * 0x1p-18f;
  const float p = fmaxf(top_p, 0.f), rest = 1.f - p;
  int first_may = kBins, first_must = kBins;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (rest * (hi_all - hi_run + off) + units >= p * lo_run) first_may = last - j;
    if (rest * (lo_all - lo_run - off) - units >= p * hi_run) first_must = last - j;
    lo_run += lo[j];
    hi_run += hi[j];
  }
  if (first_may < kBins) atomicMin(&sh.found_bin, first_may);
  if (first_must < kBins) atomicMin(&sh.found_bin2, first_must);
  __syncthreads();
}

__device__ __forceinline__ u64 candidate(float v, int index) { return (u64)key_of(v) << 32 | (uint32_t)index; }
__device__ __forceinline__ float candidate_value(u64 c) { return value_of((uint32_t)(c >> 32)); }

// Candidates are collected in the CTA first (over the cluster's counts, which have served by then): one trip to CTA 0 per
// candidate would stall its warp for a microsecond each.
__device__ __forceinline__ u64* own_list(Shared& sh) { return sh.fast.own; }
// Walks this warp's share as for_share does; the logits for which f(v) is true become candidates.  They are noted as bits
// and appended once for every 8 groups, since an append costs an atomic's round trip.
template <typename F>
__device__ __forceinline__ void collect_share(Shared& sh, const float* vals, int start, int begin, int end, F&& f) {
  const int lane = threadIdx.x & 31;
  for (int base = begin; base < end; base += 8 * 128) {
    uint32_t bits = 0;
#pragma unroll 2
    for (int g = 0; g < 8; ++g) {
      const int i = base + g * 128 + 4 * lane;
      if (base + g * 128 >= end) break;
      if (i < end) {
        const float4 v = *reinterpret_cast<const float4*>(vals + i);
        uint32_t four = 0;
        if (f(v.x)) four |= 1u;
        if (f(v.y)) four |= 2u;
        if (f(v.z)) four |= 4u;
        if (f(v.w)) four |= 8u;
        bits |= four << (4 * g);
      }
    }
    if (!__any_sync(0xffffffffu, bits != 0)) continue;
    const uint32_t mine = __popc(bits);
    const uint32_t upto = warp_scan_u32(mine);
    uint32_t at = 0;
    if (lane == 31) at = atomicAdd(&sh.own_candidates, upto);
    at = __shfl_sync(0xffffffffu, at, 31) + upto - mine;
    for (; bits != 0; bits &= bits - 1, ++at) {
      const int b = __ffs((int)bits) - 1, i = base + (b >> 2) * 128 + 4 * lane + (b & 3);
      if (at < (uint32_t)kList) own_list(sh)[at] = candidate(vals[i], start + i);
    }
  }
}
// Hands the CTA's candidates to CTA 0; the next cluster barrier makes them visible there.
__device__ void push_candidates(Shared& sh, Shared* first) {
  __syncthreads();
  const uint32_t n = sh.own_candidates;
  if (threadIdx.x == 0) sh.range[0] = atomicAdd(&first->candidates, n);
  __syncthreads();
  const uint32_t base = sh.range[0];
  for (uint32_t i = threadIdx.x; i < n; i += kThreads)
    if (base + i < (uint32_t)kList) first->fast.list[base + i] = own_list(sh)[min(i, (uint32_t)kList - 1)];
}

// CTA 0: of the candidates c (entry j of thread t is candidate 512 j + t) the one at which the running sum of `amount`, in
// ascending order, reaches `target`, which is at most the sum of all.  Histograms over ever finer ranges, 512 bins at a
// time; candidates differ (by index, if not by value), so the last range holds one.
constexpr int kPer = kList / kThreads;
__device__ u64 select_candidate(Shared& sh, const u64 (&c)[kPer], const u64 (&amount)[kPer], u64 target) {
  uint32_t* lo_sum = sh.fast.sum;  // (the counts and the CTA's own list have served)
  uint32_t* hi_sum = sh.fast.sum + kThreads;
  uint32_t* count = sh.fast.sum + 2 * kThreads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the range of the values (the indexes take all of theirs)
  uint32_t lo_key = ~0u, hi_key = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (amount[j] > 0) { lo_key = min(lo_key, (uint32_t)(c[j] >> 32)); hi_key = max(hi_key, (uint32_t)(c[j] >> 32)); }
  lo_key = __reduce_min_sync(0xffffffffu, lo_key);
  hi_key = __reduce_max_sync(0xffffffffu, hi_key);
  __syncthreads();
  if (lane == 0) { sh.warp_count[warp] = lo_key; sh.warp_high[warp] = hi_key; }
  __syncthreads();
  lo_key = __reduce_min_sync(0xffffffffu, sh.warp_count[lane % kWarps]);
  hi_key = __reduce_max_sync(0xffffffffu, (uint32_t)sh.warp_high[lane % kWarps]);
  u64 lo = (u64)lo_key << 32, hi = (u64)hi_key << 32 | 0xffffffffu;
  u64 before = 0;
  for (;;) {
    const u64 span = hi - lo;
    const int shift = max(64 - __clzll((long long)span) - 9, 0);  // span >> shift < 512
    lo_sum[threadIdx.x] = hi_sum[threadIdx.x] = count[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (amount[j] > 0 && c[j] >= lo && c[j] <= hi) {
        const int b = (int)((c[j] - lo) >> shift);
        const uint32_t add = (uint32_t)amount[j], old = atomicAdd(&lo_sum[b], add);
        atomicAdd(&hi_sum[b], (uint32_t)(amount[j] >> 32) + (old + add < old ? 1u : 0u));
        atomicAdd(&count[b], 1u);
      }
    __syncthreads();
    const u64 mine = ((u64)hi_sum[threadIdx.x] << 32) + lo_sum[threadIdx.x];
    const u64 upto = before + block_scan_u64(sh, mine);
    if (upto - mine < target && (target <= upto || threadIdx.x == kThreads - 1)) {  // (or: the search ends whatever the sums are)
      sh.found_bin = threadIdx.x;
      sh.found_weight_before = upto - mine;
      sh.found_count = count[threadIdx.x];
    }
    __syncthreads();
    const u64 first = min(lo + ((u64)sh.found_bin << shift), hi);
    if (shift == 0) return first;
    hi = min(hi, first + ((1ull << shift) - 1));
    lo = first;
    before = sh.found_weight_before;
    if (sh.found_count == 1) {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (amount[j] > 0 && c[j] >= lo && c[j] <= hi) sh.found_weight = c[j];
      __syncthreads();
      return sh.found_weight;
    }
  }
}

// CTA 0, after top-k, few candidates: each thread ranks its own against all the others, once by (value, index) with the
// weight in front of it (top-k, top-p), once among the kept ones by index (the draw).  2 x n steps of a broadcast read
// instead of two searches and a scan of a share: 8 x 32000 logits with top-k 50 and top-p took 22 us that way,
// 14 this way.
constexpr int kSmallList = 256;
__device__ void finish_small(const SampleParams& p, Shared& sh, const Row& row, int64_t i_row, int n, int k, float top_p,
                             u64 min_weight) {
  u64* weights = own_list(sh);  // (has served)
  const u64* list = sh.fast.list;
  const int t = threadIdx.x;
  const u64 c = t < n ? list[t] : ~0ull, w = t < n ? row.weight(candidate_value(c)) : 0;
  if (t < n) weights[t] = w;
  __syncthreads();
  int rank = 0;
  u64 before = 0;
  if (t < n)
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const bool less = list[j] < c;
      rank += less;
      before += less ? weights[j] : 0;
    }
  bool kept = t < n && rank < k;
  if (top_p < 1.f) {
    const u64 total = block_scan_u64(sh, kept ? w : 0);
    if (t == kThreads - 1) sh.total = total;
    __syncthreads();
    kept = kept && before < max((u64)ceil((double)fmaxf(top_p, 0.f) * (double)sh.total), 1ull);
  }
  const u64 mine = kept && w >= min_weight ? w : 0;
  const u64 total = block_scan_u64(sh, mine);
  if (t == kThreads - 1) sh.total = total;
  if (t < n) weights[t] = mine;
  __syncthreads();
  const u64 target = draw_target(p, i_row, sh.total);
  before = 0;
  if (mine > 0) {
#pragma unroll 4
    for (int j = 0; j < n; ++j) before += (uint32_t)list[j] < (uint32_t)c ? weights[j] : 0;
    if (before <= target && target < before + mine) write_token(p, i_row, (uint32_t)c, mine, sh.total);
  }
}

// CTA 0: adds the kept candidates, those up to `last` of at least min_weight, to the sums of their shares.
__device__ __forceinline__ void add_to_shares(Shared& sh, const SampleParams& p, int share, const u64 (&c)[kPer],
                                              const u64 (&w)[kPer], u64 last, u64 min_weight) {
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (c[j] <= last && w[j] >= min_weight) {
      const int index = (int)(uint32_t)c[j], cta = index / p.slice;
      uint32_t* half = reinterpret_cast<uint32_t*>(&sh.share_weight[cta * kWarps + (index - cta * p.slice) / share]);
      const uint32_t add = (uint32_t)w[j], old = atomicAdd(half, add);  // (no native 64-bit addition in shared memory)
      atomicAdd(half + 1, (uint32_t)(w[j] >> 32) + (old + add < old ? 1u : 0u));
    }
}

// CTA 0, top-p without top-k or no cut at all: share_weight holds the kept weight of every warp's share up to the
// candidates, `last` the last kept (key, index), ~0 for no cut.  Finds the share that the draw falls into and scans it
// (its logits are read again from global memory: the other CTAs are gone).
template <typename T>
__device__ void finish_shares(const SampleParams& p, Shared& sh, const Row& row, Remap remap, int64_t i_row, int n, int share,
                              u64 last, u64 min_weight) {
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
  for (int base = start; base < end; base += 2 * kThreads) {  // (one step for shares of up to 1024)
    const int i = base + 2 * threadIdx.x;
    u64 w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      w[j] = 0;
      if (i + j < end) {
        const float v = remapped(clean(widen<T>(src[i + j])), remap);
        if (candidate(v, i + j) <= last) w[j] = row.weight(v);
        if (w[j] < min_weight) w[j] = 0;
      }
    }
    const u64 to = before + block_scan_u64(sh, w[0] + w[1]), from = to - w[0] - w[1];
    if (from <= target && target < to) {
      const int j = target < from + w[0] ? 0 : 1;
      write_token(p, i_row, i + j, w[j], total);
    }
    if (threadIdx.x == kThreads - 1) sh.token_weight = to;
    __syncthreads();
    before = sh.token_weight;
    if (target < before) break;
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
  const u64 target = draw_target(p, i_row, total);
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
  sh.table[threadIdx.x] = kPowers.v[threadIdx.x];
  for (int i = threadIdx.x; i < kBins / 2; i += kThreads) sh.fast.hist[i] = 0;
  if (threadIdx.x == 0) { sh.candidates = sh.own_candidates = 0; sh.first_max = 0xffffffffu; }
  cluster_started_arrive();
  griddep_wait();
  griddep_launch_dependents();

  float temperature = p.temperature ? __ldg(p.temperature + i_row) : 1.f;
  int top_k = p.top_k ? __ldg(p.top_k + i_row) : 0;
  const float top_p = p.top_p ? __ldg(p.top_p + i_row) : 1.f;
  const float min_p = p.min_p ? __ldg(p.min_p + i_row) : 0.f;
  if (!(temperature > 0.f)) { temperature = 1.f; top_k = 1; }
  temperature = fminf(fmaxf(temperature, 1e-30f), 1e30f);
  // (NaN and values below 0 filter nothing; a weight of zero units is never kept)
  const u64 min_weight = min_p > 0.f ? max((u64)ceil((double)fminf(min_p, 1.f) * (double)(1ull << kFixed)), 1ull) : 1ull;

  const int start = min(rank * p.slice, p.vocab), len = min(p.slice, p.vocab - start);
  float mx = load_slice<T>(static_cast<const T*>(p.logits) + i_row * p.ld + start, vals, len);
  mx = warp_max(mx);
  if (lane == 0) sh.warp_max[warp] = mx;
  __syncthreads();
  cluster_started_wait();  // the row's loads lie between
  if (threadIdx.x < n) {
    for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, sh.warp_max[w]);
    cluster.map_shared_rank(&sh, threadIdx.x)->peer_max[rank] = mx;
  }
  cluster.sync();
  Row row;
  row.table = sh.table;
  float row_max = -INFINITY;
  for (int r = 0; r < n; ++r) row_max = fmaxf(row_max, sh.peer_max[r]);
  const Remap remap = row_max == INFINITY ? Remap::kInfinite
                      : row_max > -INFINITY && (double)row_max - 33.0 * (double)temperature < -3.4028234e38 ? Remap::kScale
                                                                                                            : Remap::kNone;
  if (remap != Remap::kNone) {
    for (int i = threadIdx.x; i < (len + 3) / 4 * 4; i += kThreads) vals[i] = remapped(vals[i], remap);
    row_max = remapped(row_max, remap);
    if (remap == Remap::kScale) temperature *= kRemapScale;
    __syncthreads();
  }
  row.set(row_max, temperature);
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
  const bool by_rank = top_k > 1 && top_k < p.vocab;
  if (by_rank || top_p < 1.f) {
    for_share(vals, w_begin, w_end, [&](float v, int) {
      const float b = row.biased_bin(v);
      if (b < Row::kBinEnd) atomicAdd(&sh.fast.hist[(__float_as_int(b) & 0xffff) >> 1], __float_as_int(b) & 1 ? 0x10000u : 1u);
    });
    sum_histograms(cluster, sh, n);
  }
  if (by_rank) {
    locate_rank(sh, (uint32_t)top_k);
    const int bin = sh.found_bin;
    const uint32_t count = sh.found_count;
    if (count > (uint32_t)kList) {
      slow_path<T>(cluster, p, sh, row, vals, i_row, start, len, n, rank, top_k, top_p, min_weight);
      return;
    }
    const float last_bin = Row::kBinBias + bin;
    collect_share(sh, vals, start, w_begin, w_end, [&](float v) { return row.biased_bin(v) <= last_bin; });
    push_candidates(sh, first);
    cluster.sync();
    if (rank != 0) return;
    if (count <= (uint32_t)kSmallList) {
      finish_small(p, sh, row, i_row, (int)count, top_k, top_p, min_weight);
      return;
    }
    u64 c[kPer], w[kPer], one[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = j * kThreads + threadIdx.x;
      one[j] = i < (int)count ? 1 : 0;
      c[j] = one[j] ? sh.fast.list[i] : ~0ull;
    }
    u64 last = select_candidate(sh, c, one, (u64)min((uint32_t)top_k, count));
    u64 sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      w[j] = c[j] <= last ? row.weight(candidate_value(c[j])) : 0;
      sum += w[j];
    }
    if (threadIdx.x < kMaxCluster * kWarps) sh.share_weight[threadIdx.x] = 0;
    sum = block_scan_u64(sh, sum);
    if (top_p < 1.f) {
      if (threadIdx.x == kThreads - 1) sh.total = sum;
      __syncthreads();
      last = select_candidate(sh, c, w, max((u64)ceil((double)fmaxf(top_p, 0.f) * (double)sh.total), 1ull));
    }
    add_to_shares(sh, p, share, c, w, last, min_weight);
    finish_shares<T>(p, sh, row, remap, i_row, n, share, last, min_weight);
    return;
  }
  if (top_p < 1.f) {
    locate_weight(sh, top_p, p.vocab);
    const int low = sh.found_bin, high = sh.found_bin2;
    const float low_bin = Row::kBinBias + low, high_bin = Row::kBinBias + high;
    double all = 0.0, above = 0.0, kept = 0.0;
    if (min_weight <= 1)
      collect_share(sh, vals, start, w_begin, w_end, [&](float v) {
        const float b = row.biased_bin(v);
        const double w = row.weight_d(v);
        all += w;
        if (b < low_bin) above += w;
        return b >= low_bin && b <= high_bin;
      });
    else
      collect_share(sh, vals, start, w_begin, w_end, [&](float v) {
        const float b = row.biased_bin(v);
        const double w = row.weight_d(v);
        all += w;
        if (b < low_bin) {
          above += w;
          if (w >= (double)min_weight) kept += w;
        }
        return b >= low_bin && b <= high_bin;
      });
    if (min_weight <= 1) kept = above;
    push_candidates(sh, first);
    const u64 kept_sum = warp_sum_u64((u64)kept);
    if (lane == 0) first->share_weight[rank * kWarps + warp] = kept_sum;
    const u64 all_sum = warp_sum_u64((u64)all), above_sum = warp_sum_u64((u64)above);
    if (lane == 0) { sh.warp_weight[warp] = all_sum; sh.warp_high[warp] = above_sum; }
    __syncthreads();
    if (threadIdx.x < n) {
      u64 cta_all = 0, cta_above = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) { cta_all += sh.warp_weight[w]; cta_above += sh.warp_high[w]; }
      Shared* peer = cluster.map_shared_rank(&sh, threadIdx.x);
      peer->peer_total[rank] = cta_all;
      peer->peer_above[rank] = cta_above;
      peer->peer_candidates[rank] = sh.own_candidates;
    }
    cluster.sync();
    uint32_t count = 0;
    u64 total = 0, before = 0;
    for (int r = 0; r < n; ++r) {
      count += sh.peer_candidates[r];
      total += sh.peer_total[r];
      before += sh.peer_above[r];
    }
    const u64 need = max((u64)ceil((double)fmaxf(top_p, 0.f) * (double)total), 1ull);
    if (count > (uint32_t)kList) {
      slow_path<T>(cluster, p, sh, row, vals, i_row, start, len, n, rank, top_k, top_p, min_weight);
      return;
    }
    if (rank != 0) return;
    // the last candidate whose predecessors weigh less than `need`
    u64 c[kPer], w[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = j * kThreads + threadIdx.x;
      c[j] = i < (int)count ? sh.fast.list[i] : ~0ull;
      w[j] = i < (int)count ? row.weight(candidate_value(c[j])) : 0;
    }
    const u64 last = select_candidate(sh, c, w, need - before);
    add_to_shares(sh, p, share, c, w, last, min_weight);
    finish_shares<T>(p, sh, row, remap, i_row, n, share, last, min_weight);
    return;
  }
  double kept = 0.0;
  for_share(vals, w_begin, w_end, [&](float v, int) {
    const double w = row.weight_d(v);
    kept += w >= (double)min_weight ? w : 0.0;
  });
  const u64 kept_sum = warp_sum_u64((u64)kept);
  if (lane == 0) first->share_weight[rank * kWarps + warp] = kept_sum;
  cluster.sync();
  if (rank == 0) finish_shares<T>(p, sh, row, remap, i_row, n, share, ~0ull, min_weight);
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
