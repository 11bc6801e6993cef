// Norm after a block, gate, scaled residual sum and norm before the next block in one pass:
//
//   h[i,j] = alpha * x[i,j] + gate[i / gate_rows, j] * Post(y[i,:])[j]
//   n[i,j] = Pre(h[i,:])[j]
//
// with Post and Pre nothing, RMSNorm or LayerNorm (biased variance, eps inside the root).  HBM-bound: x and y are read
// once, h and n written once (8 bytes per element for bf16 streams, 12 with an fp32 residual stream), and the row
// stays in registers from the first load to the last store.  Statistics are fp32; LayerNorm's second moment is taken
// about the mean (no E[v^2] - mean^2 cancellation), which costs a reduction more than RMSNorm; each reduction is a
// warp shuffle tree and, for rows that several warps share, one barrier.  Only h and n are rounded, and n is computed
// from the unrounded h.
//
// A thread holds UNITS groups of 8 elements.  Rows of up to 512 columns take a warp, longer ones a CTA.  What holds long
// runs of rows back is the latency of a row's reductions at 32 warps per SM (IPC 1.4), and the parameter vectors, which
// come through an L1 that the rows flush (16384 x 4096, fp32 stream, RMSNorm and LayerNorm: 151 us, 129 of them without the
// vectors, 127 without the norms).  For bf16 streams with many rows, persistent CTAs of several row groups have each
// group's next row copied to shared memory in bulk while the current one is worked on, and keep the vectors there.
#include <cmath>

#include "pd_common.cuh"
#include "sm100_ptx.cuh"

namespace pd {
namespace {

struct NormParams {
  const void *y, *x, *gate;
  const float *post_gamma, *post_beta, *pre_gamma, *pre_beta;
  void *h, *n;
  int64_t rows, gate_rows;
  int cols, post_norm, pre_norm;
  float alpha, eps;
  unsigned long long wait_limit_ns;  // (of the kernel that prefetches rows, as is the next one)
  int withhold_loads;                // test switch: rows are not requested, and the first wait for one runs out
};

struct Raw8f { float4 a, b; };
// 8 elements as they lie in memory, and as floats
__device__ __forceinline__ uint4 load_raw8(const __nv_bfloat16* p) { return __ldcs(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ Raw8f load_raw8(const float* p) {
  return {__ldcs(reinterpret_cast<const float4*>(p)), __ldcs(reinterpret_cast<const float4*>(p) + 1)};
}
__device__ __forceinline__ void widen8(const uint4& r, float (&v)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen8(const Raw8f& r, float (&v)[8]) {
  v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w; v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&t);
  }
  __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void load_vec8(const float* p, float (&v)[8]) {  // a parameter vector: stays cached
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ uint4 load_gate8(const __nv_bfloat16* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ Raw8f load_gate8(const float* p) {
  return {__ldg(reinterpret_cast<const float4*>(p)), __ldg(reinterpret_cast<const float4*>(p) + 1)};
}

// Sums of two values over the row's threads.
template <int NW>
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 (*scratch)[NW], int slot) {
  a = warp_sum(a);
  b = warp_sum(b);
  if constexpr (NW == 1) return make_float2(a, b);
  if ((threadIdx.x & 31) == 0) scratch[slot][threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  float2 r = scratch[slot][0];
#pragma unroll
  for (int w = 1; w < NW; ++w) { r.x += scratch[slot][w].x; r.y += scratch[slot][w].y; }
  return r;
}

// v <- norm(v) over the row that THREADS threads hold, elements beyond the row left alone.
template <int UNITS, int THREADS>
__device__ __forceinline__ void norm_row(float (&v)[UNITS][8], int t, int units, int kind, float inv_cols, float eps,
                                         const float* gamma, const float* beta, float2 (*scratch)[THREADS / 32], int& slot) {
  constexpr int NW = THREADS / 32;
  if (kind == PD_NORM_NONE) return;
  float shift = 0.f;
  if (kind == PD_NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
      if (t + i * THREADS < units)
        sum += ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3])) + ((v[i][4] + v[i][5]) + (v[i][6] + v[i][7]));
    shift = block_sum2<NW>(sum, 0.f, scratch, slot).x * inv_cols;
    slot ^= 1;
  }
  float sum = 0.f, q = 0.f;
#pragma unroll
  for (int i = 0; i < UNITS; ++i)
    if (t + i * THREADS < units)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = v[i][j] - shift;
        v[i][j] = d;
        sum += d;
        q = fmaf(d, d, q);
      }
  const float2 m = block_sum2<NW>(sum, q, scratch, slot);
  slot ^= 1;
  const float rest = kind == PD_NORM_LAYER ? m.x * inv_cols : 0.f;
  const float rstd = rsqrtf(fmaxf(m.y * inv_cols - rest * rest, 0.f) + eps);
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const int c = t + i * THREADS;
    if (c < units) {
      float gm[8];
      if (gamma) {
        load_vec8(gamma + 8 * c, gm);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - rest) * (rstd * gm[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - rest) * rstd;
      }
      if (kind == PD_NORM_LAYER && beta) {
        load_vec8(beta + 8 * c, gm);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += gm[j];
      }
    }
  }
}

// 1024 threads per SM at 64 registers: left alone, the compiler takes 80 to 98 and two or three rows of 4096 columns are in
// flight per SM instead of four (16384 x 4096: 171 against 151 us; at 48 registers it spills, 177).  Rows beyond 8192
// columns, 32 elements to a thread, need the registers more.
template <typename TX, typename TY, int UNITS, int THREADS_PER_ROW, int THREADS_PER_CTA>
__global__ void __launch_bounds__(THREADS_PER_CTA, UNITS > 2 ? 1 : 1024 / THREADS_PER_CTA)
norm_gate_residual_rows_in_registers(const NormParams p) {
  constexpr int ROWS = THREADS_PER_CTA / THREADS_PER_ROW;
  __shared__ float2 scratch[2][THREADS_PER_ROW / 32];
  const int t = threadIdx.x % THREADS_PER_ROW;
  const int units = p.cols >> 3;
  const float inv_cols = 1.0f / (float)p.cols;
  griddep_wait();
  griddep_launch_dependents();
  int slot = 0;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS_PER_ROW; row < p.rows;
       row += (int64_t)gridDim.x * ROWS) {
    const TY* y = static_cast<const TY*>(p.y) + row * p.cols;
    const TX* x = static_cast<const TX*>(p.x) + row * p.cols;
    decltype(load_raw8(y)) ry[UNITS];
    decltype(load_raw8(x)) rx[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
      if (t + i * THREADS_PER_ROW < units) ry[i] = load_raw8(y + 8 * (t + i * THREADS_PER_ROW));
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
      if (t + i * THREADS_PER_ROW < units) rx[i] = load_raw8(x + 8 * (t + i * THREADS_PER_ROW));
    float v[UNITS][8];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) widen8(ry[i], v[i]);
    norm_row<UNITS, THREADS_PER_ROW>(v, t, units, p.post_norm, inv_cols, p.eps, p.post_gamma, p.post_beta, scratch, slot);
    const TY* gate = p.gate ? static_cast<const TY*>(p.gate) + (row / p.gate_rows) * p.cols : nullptr;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int c = t + i * THREADS_PER_ROW;
      if (c < units) {
        float xv[8];
        widen8(rx[i], xv);
        if (gate) {
          float gv[8];
          widen8(load_gate8(gate + 8 * c), gv);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j], gv[j], p.alpha * xv[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = fmaf(p.alpha, xv[j], v[i][j]);
        }
        if (p.h) store8(static_cast<TX*>(p.h) + row * p.cols + 8 * c, v[i]);
      }
    }
    if (p.n) {
      norm_row<UNITS, THREADS_PER_ROW>(v, t, units, p.pre_norm, inv_cols, p.eps, p.pre_gamma, p.pre_beta, scratch, slot);
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int c = t + i * THREADS_PER_ROW;
        if (c < units) store8(static_cast<TY*>(p.n) + row * p.cols + 8 * c, v[i]);
      }
    }
  }
}

// ---- many rows: persistent CTAs, rows prefetched -------------------------------------------
constexpr int kTimeoutNorm = 321;  // left in the device status word when a row does not arrive

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
// Barrier of one row group (up to sixteen: group 0 takes the barrier of __syncthreads, which is not called any more then);
// true if every thread of the group says so.
template <int THREADS>
__device__ __forceinline__ bool group_all(int group, bool yes) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 q, %1, 0;\n"
      "bar.red.and.pred p, %2, %3, q;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(r)
      : "r"(yes ? 1u : 0u), "r"(group), "n"(THREADS)
      : "memory");
  return r != 0;
}
template <int THREADS>
__device__ __forceinline__ float2 group_sum2(int group, float a, float b, float2* scratch) {
  a = warp_sum(a);
  b = warp_sum(b);
  if ((threadIdx.x & 31) == 0) scratch[(threadIdx.x % THREADS) >> 5] = make_float2(a, b);
  asm volatile("bar.sync %0, %1;" ::"r"(group), "n"(THREADS) : "memory");
  float2 r = scratch[0];
#pragma unroll
  for (int w = 1; w < THREADS / 32; ++w) { r.x += scratch[w].x; r.y += scratch[w].y; }
  return r;
}
// 8 elements of a parameter vector kept as two planes of float4 (unit c: plane 0 entry c, plane 1 entry c), which reads
// without bank conflicts.
__device__ __forceinline__ void planes8(const float4* planes, int units, int c, float (&v)[8]) {
  const float4 a = planes[c], b = planes[units + c];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

constexpr int kPrefetchThreads = 1024, kPrefetchUnits = 2;

// T threads per row, 1024 / T row groups per CTA, one CTA per SM.
template <typename TX, typename TY, int T>
__global__ void __launch_bounds__(kPrefetchThreads, 1) norm_gate_residual_rows_prefetched(const NormParams p, int* status) {
  constexpr int kGroups = kPrefetchThreads / T, UNITS = kPrefetchUnits;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float2 scratch[kGroups][4][T / 32];  // two sums of either norm: a group's warps may be one sum apart
  __shared__ __align__(8) uint64_t bars[kGroups];
  __shared__ int abort_flag;
  const int group = threadIdx.x / T, t = threadIdx.x % T;
  const int units = p.cols >> 3;
  const float inv_cols = 1.0f / (float)p.cols;
  const uint32_t y_bytes = (uint32_t)p.cols * sizeof(TY), x_bytes = (uint32_t)p.cols * sizeof(TX);
  uint8_t* ys = smem + (size_t)group * (y_bytes + x_bytes);
  uint8_t* xs = ys + y_bytes;
  float4* planes = reinterpret_cast<float4*>(smem + (size_t)kGroups * (y_bytes + x_bytes));
  const uint32_t bar = sm100::smem_u32(&bars[group]);
  if (threadIdx.x == 0) {
    for (int g = 0; g < kGroups; ++g) sm100::mbar_init(sm100::smem_u32(&bars[g]), 1);
    abort_flag = 0;
    sm100::fence_barrier_init();
    sm100::fence_proxy_async_smem();
  }
  griddep_wait();
  griddep_launch_dependents();
  // the parameter vectors that the norms use, in this order
  const float4* vec[4] = {nullptr, nullptr, nullptr, nullptr};
  {
    const float* src[4] = {p.post_norm != PD_NORM_NONE ? p.post_gamma : nullptr, p.post_norm == PD_NORM_LAYER ? p.post_beta : nullptr,
                           p.pre_norm != PD_NORM_NONE && p.n ? p.pre_gamma : nullptr,
                           p.pre_norm == PD_NORM_LAYER && p.n ? p.pre_beta : nullptr};
    float4* at = planes;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (src[k]) {
        vec[k] = at;
        for (int c = threadIdx.x; c < 2 * units; c += kPrefetchThreads)
          at[(c & 1) * units + (c >> 1)] = __ldg(reinterpret_cast<const float4*>(src[k]) + c);
        at += 2 * units;
      }
  }
  __syncthreads();

  const int64_t step = (int64_t)gridDim.x * kGroups;
  int64_t row = (int64_t)blockIdx.x * kGroups + group;
  auto fetch = [&](int64_t r) {  // by the group's first thread
    if (p.withhold_loads) return;
    sm100::mbar_arrive_expect_tx(bar, y_bytes + x_bytes);
    bulk_load(sm100::smem_u32(ys), static_cast<const TY*>(p.y) + r * p.cols, y_bytes, bar);
    bulk_load(sm100::smem_u32(xs), static_cast<const TX*>(p.x) + r * p.cols, x_bytes, bar);
  };
  if (t == 0 && row < p.rows) fetch(row);
  uint32_t parity = 0;
  // v <- norm(v)
  auto norm = [&](float (&v)[UNITS][8], int kind, const float4* gamma, const float4* beta, float2 (*sums)[T / 32]) {
    if (kind == PD_NORM_NONE) return;
    float shift = 0.f;
    if (kind == PD_NORM_LAYER) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < UNITS; ++i)
        if (t + i * T < units)
          sum += ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3])) + ((v[i][4] + v[i][5]) + (v[i][6] + v[i][7]));
      shift = group_sum2<T>(group, sum, 0.f, sums[0]).x * inv_cols;
    }
    float sum = 0.f, q = 0.f;
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
      if (t + i * T < units)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = v[i][j] - shift;
          v[i][j] = d;
          sum += d;
          q = fmaf(d, d, q);
        }
    const float2 m = group_sum2<T>(group, sum, q, sums[1]);
    const float rest = kind == PD_NORM_LAYER ? m.x * inv_cols : 0.f;
    const float rstd = rsqrtf(fmaxf(m.y * inv_cols - rest * rest, 0.f) + p.eps);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int c = t + i * T;
      if (c < units) {
        float w[8];
        if (gamma) {
          planes8(gamma, units, c, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - rest) * (rstd * w[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - rest) * rstd;
        }
        if (beta) {
          planes8(beta, units, c, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] += w[j];
        }
      }
    }
  };
  for (; row < p.rows; row += step, parity ^= 1u) {
    const bool here = sm100::mbar_wait(bar, parity, &abort_flag, status, kTimeoutNorm, p.wait_limit_ns);
    decltype(load_raw8(static_cast<const TX*>(nullptr))) rx[UNITS];
    float v[UNITS][8];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int c = t + i * T;
      if (c < units) {
        widen8(*(reinterpret_cast<const decltype(load_raw8(static_cast<const TY*>(nullptr)))*>(ys) + c), v[i]);
        rx[i] = *(reinterpret_cast<const decltype(load_raw8(static_cast<const TX*>(nullptr)))*>(xs) + c);
      }
    }
    // every thread has its part in registers (or one has waited in vain): the buffer is free for the next row
    if (!group_all<T>(group, here)) {
      // leave no copy in flight: give it a short time to land
      volatile int never = 0;
      sm100::mbar_wait(bar, parity, &never, nullptr, 0, 20000000ull);
      break;
    }
    if (t == 0 && row + step < p.rows) fetch(row + step);
    norm(v, p.post_norm, vec[0], vec[1], scratch[group]);
    const TY* gate = p.gate ? static_cast<const TY*>(p.gate) + (row / p.gate_rows) * p.cols : nullptr;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int c = t + i * T;
      if (c < units) {
        float xv[8];
        widen8(rx[i], xv);
        if (gate) {
          float gv[8];
          widen8(load_gate8(gate + 8 * c), gv);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j], gv[j], p.alpha * xv[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = fmaf(p.alpha, xv[j], v[i][j]);
        }
        if (p.h) store8(static_cast<TX*>(p.h) + row * p.cols + 8 * c, v[i]);
      }
    }
    if (p.n) {
      norm(v, p.pre_norm, vec[2], vec[3], scratch[group] + 2);
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int c = t + i * T;
        if (c < units) store8(static_cast<TY*>(p.n) + row * p.cols + 8 * c, v[i]);
      }
    }
  }
}

__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(float v) { return v; }

// Any length and alignment: a CTA per row that reads the row again for every statistic (from L2).
// Columns are counted in 64 bits: a thread's step behind the end of a row of 2^31 - 1 does not fit 32.
// h is computed once for every pass over the row, with its roundings written out, so that the passes agree on it: contracted
// differently they were a step apart, which LayerNorm of a row of one value multiplies by 1 / sqrt(eps).
// A thread adds runs of 64 terms in single precision (off by 2^-18 at most) and the runs in double: one running sum is off by
// 7e-5 over the 16384 terms of 4 million equal columns.
template <typename TX, typename TY>
__global__ void __launch_bounds__(256) norm_gate_residual_generic(const NormParams p) {
  constexpr int kRun = 64 * 256;
  __shared__ float2 scratch[2][8];
  griddep_wait();
  griddep_launch_dependents();
  int slot = 0;
  const float inv_cols = 1.0f / (float)p.cols;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const TY* y = static_cast<const TY*>(p.y) + row * p.cols;
    const TX* x = static_cast<const TX*>(p.x) + row * p.cols;
    const TY* gate = p.gate ? static_cast<const TY*>(p.gate) + (row / p.gate_rows) * p.cols : nullptr;
    auto stats = [&](int kind, auto&& value, float& mean, float& rstd) {
      mean = 0.f;
      rstd = 1.f;
      if (kind == PD_NORM_NONE) return;
      float shift = 0.f;
      if (kind == PD_NORM_LAYER) {
        double s = 0.0;
        for (int64_t j = threadIdx.x; j < p.cols;) {
          const int64_t end = j + kRun < p.cols ? j + kRun : p.cols;
          float run = 0.f;
          for (; j < end; j += 256) run += value(j);
          s += run;
        }
        shift = block_sum2<8>((float)s, 0.f, scratch, slot).x * inv_cols;
        slot ^= 1;
      }
      double s = 0.0, q = 0.0;
      for (int64_t j = threadIdx.x; j < p.cols;) {
        const int64_t end = j + kRun < p.cols ? j + kRun : p.cols;
        float run_s = 0.f, run_q = 0.f;
        for (; j < end; j += 256) {
          const float d = value(j) - shift;
          run_s += d;
          run_q = fmaf(d, d, run_q);
        }
        s += run_s;
        q += run_q;
      }
      const float2 m = block_sum2<8>((float)s, (float)q, scratch, slot);
      slot ^= 1;
      const float rest = kind == PD_NORM_LAYER ? m.x * inv_cols : 0.f;
      mean = shift + rest;
      rstd = rsqrtf(fmaxf(m.y * inv_cols - rest * rest, 0.f) + p.eps);
    };
    auto affine = [&](int kind, float v, float mean, float rstd, const float* gamma, const float* beta, int64_t j) {
      if (kind == PD_NORM_NONE) return v;
      v = __fmul_rn(v - mean, __fmul_rn(rstd, gamma ? gamma[j] : 1.f));
      return kind == PD_NORM_LAYER && beta ? __fadd_rn(v, beta[j]) : v;
    };
    float post_mean, post_rstd, pre_mean = 0.f, pre_rstd = 1.f;
    stats(p.post_norm, [&](int64_t j) { return widen(y[j]); }, post_mean, post_rstd);
    auto h = [&](int64_t j) {
      const float v = affine(p.post_norm, widen(y[j]), post_mean, post_rstd, p.post_gamma, p.post_beta, j);
      return gate ? __fmaf_rn(v, widen(gate[j]), __fmul_rn(p.alpha, widen(x[j]))) : __fmaf_rn(p.alpha, widen(x[j]), v);
    };
    if (p.n) stats(p.pre_norm, h, pre_mean, pre_rstd);
    for (int64_t j = threadIdx.x; j < p.cols; j += 256) {
      const float v = h(j);
      const float n = affine(p.pre_norm, v, pre_mean, pre_rstd, p.pre_gamma, p.pre_beta, j);
      if (p.h) store_out1(static_cast<TX*>(p.h), row * p.cols + j, v);
      if (p.n) store_out1(static_cast<TY*>(p.n), row * p.cols + j, n);
    }
  }
}

template <typename TX, typename TY, int UNITS, int THREADS, int CTA = THREADS>
void launch_rows(const NormParams& p, cudaStream_t s) {
  constexpr int kRows = CTA / THREADS;
  const int64_t ctas = (p.rows + kRows - 1) / kRows;
  const int grid = (int)(ctas < 0x7fffffff ? ctas : 0x7fffffff);
  launch_pdl(norm_gate_residual_rows_in_registers<TX, TY, UNITS, THREADS, CTA>, dim3(grid), dim3(CTA), 0, s, p);
}

// Shared memory of the prefetching kernel: a row of x and y (bf16) for every group of t threads, and the vectors in use.
int prefetch_smem(const NormParams& p, int t) {
  int vectors = 0;
  if (p.post_norm != PD_NORM_NONE) vectors += (p.post_gamma != nullptr) + (p.post_norm == PD_NORM_LAYER && p.post_beta != nullptr);
  if (p.pre_norm != PD_NORM_NONE) vectors += (p.pre_gamma != nullptr) + (p.pre_norm == PD_NORM_LAYER && p.pre_beta != nullptr);
  return kPrefetchThreads / t * p.cols * 4 + vectors * p.cols * 4;
}
constexpr int kPrefetchMaxSmem = 222 * 1024;
constexpr int kPrefetchMinRows = 3;  // rows of every group

template <typename TX, typename TY, int T>
pd_status launch_prefetched(const NormParams& p, cudaStream_t s) {
  static PerDeviceFlag smem_allowed;
  if (pd_status st = allow_dynamic_smem(norm_gate_residual_rows_prefetched<TX, TY, T>, kPrefetchMaxSmem, smem_allowed); st != PD_OK) return st;
  int* status = device_status_ptr();
  if (!status) return PD_ERR_CUDA;
  logf("norm gate residual norm %lld x %d: %d rows in flight per SM, the next ones prefetched", (long long)p.rows, p.cols, kPrefetchThreads / T);
  launch_pdl(norm_gate_residual_rows_prefetched<TX, TY, T>, dim3(sm_count()), dim3(kPrefetchThreads),
             prefetch_smem(p, T), s, p, status);
  return check_launch();
}

template <typename TX, typename TY>
pd_status launch(const NormParams& p, cudaStream_t s) {
  const bool vec_ok = p.cols % 8 == 0 && p.cols <= 32768 && aligned16(p.y) && aligned16(p.x) && aligned16(p.gate) &&
                      aligned16(p.h) && aligned16(p.n) && aligned16(p.post_gamma) && aligned16(p.post_beta) &&
                      aligned16(p.pre_gamma) && aligned16(p.pre_beta);
  // Measured (16384 rows, RMSNorm twice, single calls, us prefetched / not): bf16 streams, 4096 columns 96 / 109, 8192 columns
  // 209 / 234, 1024 columns 27 / 28; with a gate for every row 141 / 141 (4096) and 293 / 305 (8192).  An fp32 stream, with gates
  // and a LayerNorm, took 157 / 153 (160 in long runs), so not there.  1184 rows of 4096 columns: 11.9 / 12.2.
  if constexpr (sizeof(TX) + sizeof(TY) == 4) {
    if (vec_ok && p.cols > 1024 && p.cols <= 8192) {
      const int t = p.cols <= 2048 ? 128 : p.cols <= 4096 ? 256 : 512;
      if (p.rows >= kPrefetchMinRows * (int64_t)(kPrefetchThreads / t) * sm_count() && prefetch_smem(p, t) <= kPrefetchMaxSmem)
        return t == 128 ? launch_prefetched<TX, TY, 128>(p, s) : t == 256 ? launch_prefetched<TX, TY, 256>(p, s)
                                                                         : launch_prefetched<TX, TY, 512>(p, s);
    }
  }
  logf("norm gate residual norm %lld x %d: %s", (long long)p.rows, p.cols,
       !vec_ok ? "scalar path (unaligned, ragged or very long rows)" : p.cols <= 512 ? "one warp per row, row in registers"
       : "one CTA per row, row in registers");
  if (!vec_ok) {
    const int64_t cap = (int64_t)sm_count() * 8;
    launch_pdl(norm_gate_residual_generic<TX, TY>, dim3((unsigned)(p.rows < cap ? p.rows : cap)), dim3(256), 0, s, p);
  } else if (p.cols <= 256) launch_rows<TX, TY, 1, 32, 64>(p, s);
  else if (p.cols <= 512) launch_rows<TX, TY, 2, 32, 64>(p, s);
  else if (p.cols <= 1024) launch_rows<TX, TY, 2, 64>(p, s);
  else if (p.cols <= 2048) launch_rows<TX, TY, 2, 128>(p, s);
  else if (p.cols <= 4096) launch_rows<TX, TY, 2, 256>(p, s);
  else if (p.cols <= 8192) launch_rows<TX, TY, 2, 512>(p, s);
  else if (p.cols <= 16384) launch_rows<TX, TY, 4, 512>(p, s);
  else launch_rows<TX, TY, 4, 1024>(p, s);
  return check_launch();
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_norm_gate_residual_norm(const pd_norm_gate_residual_desc* desc, const void* y, const void* x,
                                                const void* gate, const float* post_gamma, const float* post_beta,
                                                const float* pre_gamma, const float* pre_beta, void* h, void* n,
                                                cudaStream_t stream) {
  if (!desc) return PD_ERR_NULL_POINTER;
  const pd_norm_gate_residual_desc& d = *desc;
  if (d.rows < 0 || d.cols <= 0 || d.cols > 0x7fffffff || !(d.eps >= 0.f) || !std::isfinite(d.alpha)) return PD_ERR_BAD_SHAPE;
  if (gate && d.gate_rows < 1) return PD_ERR_BAD_SHAPE;
  auto is_dtype = [](int t) { return t == PD_BF16 || t == PD_F32; };
  auto is_norm = [](int k) { return k >= PD_NORM_NONE && k <= PD_NORM_LAYER; };
  if (!is_dtype(d.x_dtype) || !is_dtype(d.y_dtype) || !is_norm(d.post_norm) || !is_norm(d.pre_norm)) return PD_ERR_BAD_SHAPE;
  if (d.rows == 0) return PD_OK;  // (an empty tensor's pointers may be null)
  if (!y || !x || (!h && !n)) return PD_ERR_NULL_POINTER;
  auto bits = [](const void* q) { return reinterpret_cast<uintptr_t>(q); };
  const uintptr_t xb = bits(x) | bits(h), yb = bits(y) | bits(n) | bits(gate);
  if ((xb & (d.x_dtype == PD_F32 ? 3u : 1u)) || (yb & (d.y_dtype == PD_F32 ? 3u : 1u)) ||
      ((bits(post_gamma) | bits(post_beta) | bits(pre_gamma) | bits(pre_beta)) & 3u))
    return PD_ERR_ALIGNMENT;
  if (pd_status st = pd::require_sm100(); st != PD_OK) return st;
  pd::NormParams p{y, x, gate, post_gamma, post_beta, pre_gamma, pre_beta, h, n, d.rows, gate ? d.gate_rows : 1,
                   (int)d.cols, d.post_norm, d.pre_norm, d.alpha, d.eps, pd::debug_wait_limit_ns(), pd::debug_withhold_loads()};
  if (d.x_dtype == PD_BF16)
    return d.y_dtype == PD_BF16 ? pd::launch<__nv_bfloat16, __nv_bfloat16>(p, stream) : pd::launch<__nv_bfloat16, float>(p, stream);
  return d.y_dtype == PD_BF16 ? pd::launch<float, __nv_bfloat16>(p, stream) : pd::launch<float, float>(p, stream);
}
