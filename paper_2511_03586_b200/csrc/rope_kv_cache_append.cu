// Rotates the new tokens' queries and keys by their positions and appends keys and values to the paged cache, as bf16 or
// in 8 bits with a scale for each block of tokens and head:
//
//   theta_i = p * inv_freq[i],   (a, b) -> amplitude * (a cos theta_i - b sin theta_i, a sin theta_i + b cos theta_i)
//
// for the pairs (a, b) = (x[i], x[i + R/2]) or, interleaved, (x[2i], x[2i + 1]) of a head's first R elements.
//
// Angles: far positions make p * inv_freq as large as 10^6 radians, where fp32 keeps two digits of the angle.  The number of
// turns p * inv_freq / 2 pi is formed in 64 bits (p has 31 bits, inv_freq 24: off by 2^-52 of itself), its whole part dropped,
// and the rest, at most half a turn, goes through sincospif.  A warp does that once per token for all its heads.
//
// Bound: HBM for prompts.  Every element of q, k and v is read once and written once (the rotation is 6 operations on 4 bytes);
// a decode batch is one launch and a chain of four dependent loads.
//
// The 8-bit cache: a block's scale is its largest magnitude over the top of the type, so all of its new tokens have to be seen
// before the first is rounded.  A CTA takes one block of one sequence and up to eight heads of K or of V of it, a warp or, for blocks
// of more than 256 units of 8 elements (16 tokens of 128), several to a head; they hold the block in registers between the two passes as
// long as it has at most 2048 units, and read it again, from the L2 cache, beyond that.  Values are rounded once, from the rotated fp32
// ones.  A block that held older tokens keeps its scale unless a new token exceeds it; then the older values are rounded again,
// to the larger step.
//   8 x up to 2048 tokens, 32/8 heads of 128, in long runs: 67 us into a bf16 cache (73 % of the copy rate), 73 into an e4m3 cache with blocks
//   of 32 (61 %).
#include "cache_q8.cuh"

namespace pd {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kUnit = 8;         // elements that one lane handles at a time: four pairs, or eight elements that are not rotated
constexpr int kHeld = 8;         // units a lane holds between the passes of the 8-bit form
constexpr int kGroup = 32 * kHeld;  // and a warp
constexpr int kMaxDim = 256;
constexpr int kMaxPairs = kMaxDim / 2;
constexpr int kMaxIndex = 1 << 30;

struct RopeParams {
  const __nv_bfloat16 *q, *k_new, *v_new;
  __nv_bfloat16* q_out;
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  const float* inv_freq;
  const int32_t *block_table, *cu_q, *kv_len;
  int64_t ld_q, ld_q_out, ld_new, page_stride, slot_stride, head_stride;  // in elements
  paged::Scales scales;
  float amplitude;
  int rotary, interleaved;
  int batch, tokens, heads_q, heads_kv, head_dim;
  int num_pages, page_size, max_pages;
  int parts;           // warps that share a token
  int warps_a_head;    // 8-bit form: warps that share a head of a block
  int rounds;          // 8-bit form: CTAs that share a block, each up to kWarps / warps_a_head heads of K or of V
  int64_t block_ctas;  // 8-bit form: CTAs in front of the ones that rotate queries
};

// cos and sin of position `pos` times inv_freq[i], times the amplitude.
__device__ __forceinline__ float2 turn_of(const RopeParams& p, int pos, int i) {
  const double turns = (double)pos * (double)__ldg(p.inv_freq + i) * 0.15915494309189533577;  // 1 / 2 pi
  float s, c;
  sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
  return make_float2(c * p.amplitude, s * p.amplitude);
}

// Unit u of a head: its eight elements lie at `first` and, for split pairs, four at each of `first` and `second`.
struct Place {
  int first, second;
  bool rotated, split;
};
__device__ __forceinline__ Place place_of(const RopeParams& p, int u) {
  Place at;
  at.rotated = u * kUnit < p.rotary;
  at.split = at.rotated && !p.interleaved;
  at.first = at.split ? 4 * u : kUnit * u;
  at.second = at.first + (at.split ? p.rotary / 2 : 4);
  return at;
}
__device__ __forceinline__ uint4 load_unit(const __nv_bfloat16* head, const Place& at) {
  if (!at.split) return __ldcs(reinterpret_cast<const uint4*>(head + at.first));
  const uint2 a = __ldcs(reinterpret_cast<const uint2*>(head + at.first)), b = __ldcs(reinterpret_cast<const uint2*>(head + at.second));
  return make_uint4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float2 bf16_pair(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
// The unit's elements in fp32, rotated by the four turns behind `turns` (of this unit).
__device__ __forceinline__ void rotate_unit(uint4 raw, const Place& at, const float2* turns, float (&x)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = bf16_pair(w[i]);
    x[2 * i] = v.x;
    x[2 * i + 1] = v.y;
  }
  if (!at.rotated) return;
  auto turn = [](float& a, float& b, float2 t) {
    const float a0 = a, b0 = b;
    a = fmaf(a0, t.x, -(b0 * t.y));
    b = fmaf(a0, t.y, b0 * t.x);
  };
  if (at.split) {  // (two loops, so that the elements stay in registers)
#pragma unroll
    for (int i = 0; i < 4; ++i) turn(x[i], x[i + 4], turns[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) turn(x[2 * i], x[2 * i + 1], turns[i]);
  }
}
__device__ __forceinline__ void store_unit(__nv_bfloat16* head, const Place& at, const float (&x)[8]) {
  const uint4 v = make_uint4(paged::pack_bf16(x[0], x[1]), paged::pack_bf16(x[2], x[3]), paged::pack_bf16(x[4], x[5]), paged::pack_bf16(x[6], x[7]));
  if (!at.split) {
    *reinterpret_cast<uint4*>(head + at.first) = v;
  } else {
    *reinterpret_cast<uint2*>(head + at.first) = make_uint2(v.x, v.y);
    *reinterpret_cast<uint2*>(head + at.second) = make_uint2(v.z, v.w);
  }
}

// A sequence's new tokens: rows [q0, q0 + n), the first at position pos0 (negative where kv_len is short of n).
struct NewTokens {
  int q0, n, pos0;
};
__device__ __forceinline__ NewTokens new_tokens(const RopeParams& p, int from, int to, int length) {
  NewTokens s;
  s.q0 = min(max(from, 0), p.tokens);
  s.n = min(max(to, s.q0), p.tokens) - s.q0;
  s.pos0 = max(length, 0) - s.n;
  return s;
}
// The number of sequences b >= 0 in front of the first one for which inside(b, cu_q[b], cu_q[b + 1]) is false (it holds for leading
// ones only), and in `s` the tokens of sequence `that number - back`.  A warp.  Up to 128 sequences are looked at at once, with
// their lengths, so that a decode batch waits for one round of loads instead of three.
template <typename F>
__device__ __forceinline__ int find_tokens(const RopeParams& p, int back, NewTokens& s, F inside) {
  const int lane = threadIdx.x & 31;
  int b;
  if (p.batch <= 128) {
    int from[4], to[4], length[4], n = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = lane + 32 * k;
      const bool there = i < p.batch;
      from[k] = there ? __ldg(p.cu_q + i) : 0;
      to[k] = there ? __ldg(p.cu_q + i + 1) : 0;
      length[k] = there ? __ldg(p.kv_len + i) : 0;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) n += __popc(__ballot_sync(0xffffffffu, lane + 32 * k < p.batch && inside(lane + 32 * k, from[k], to[k])));
    b = n;
    const int at = min(max(b - back, 0), 127);
    int f = 0, e = 0, l = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int f1 = __shfl_sync(0xffffffffu, from[k], at & 31), e1 = __shfl_sync(0xffffffffu, to[k], at & 31), l1 = __shfl_sync(0xffffffffu, length[k], at & 31);
      if (at >> 5 == k) { f = f1; e = e1; l = l1; }
    }
    s = new_tokens(p, f, e, l);
    return b;
  }
  int lo = 0, hi = p.batch;  // the answer lies in [lo, hi]
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const int i = lo + lane * step;
    const unsigned yes = __ballot_sync(0xffffffffu, i < hi && inside(i, __ldg(p.cu_q + min(i, p.batch - 1)), __ldg(p.cu_q + min(i, p.batch - 1) + 1)));
    const int k = __popc(yes);
    if (k == 0) break;
    const int next = lo + (k - 1) * step + 1;
    hi = min(lo + k * step, hi);
    lo = next;
  }
  b = lo;
  const int at = min(max(b - back, 0), p.batch - 1);
  s = new_tokens(p, __ldg(p.cu_q + at), __ldg(p.cu_q + at + 1), __ldg(p.kv_len + at));
  return b;
}
__device__ __forceinline__ int page_at(const RopeParams& p, int b, int pos) {
  const int i = pos / p.page_size;
  if (i >= p.max_pages) return -1;
  const int page = __ldg(p.block_table + (int64_t)b * p.max_pages + i);
  return (unsigned)page < (unsigned)p.num_pages ? page : -1;
}

// Units of a token's heads, `steps` of them for this lane, src_step and dst_step elements apart: read, rotated by the turns of its
// unit (ROTATE; else copied), and written.  AHEAD loads are under way together.
template <bool ROTATE, int AHEAD>
__device__ __forceinline__ void turn_units(const __nv_bfloat16* src, int src_step, __nv_bfloat16* dst, int64_t dst_step, int steps, const Place& at,
                                           const float2 (&turn)[4]) {
  for (; steps > 0; steps -= AHEAD, src += AHEAD * src_step, dst += AHEAD * dst_step) {
    uint4 raw[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (j < steps) raw[j] = load_unit(src + j * src_step, at);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (j < steps) {
        if (ROTATE && at.rotated) {
          float x[8];
          rotate_unit(raw[j], at, turn, x);
          store_unit(dst + j * dst_step, at, x);
        } else {
          *reinterpret_cast<uint4*>(dst + j * dst_step + at.first) = raw[j];
        }
      }
    }
  }
}

// `part` of the heads of token t: queries to q_out and, for a bf16 cache (CACHE), keys and values to their slot.  A warp.
//   Where the units of a head divide 32 (head_dim 32, 64, 128 or 256) a lane has the same unit of every head it comes to: its place and
//   its turns stay in registers, and from step to step only the head changes.  (With units found by division for every step, and
//   turns read from shared memory, 8 x 2048 tokens took 76 us single; now 65, where more loads ahead cost more than they bring, 88 with six.)
template <bool CACHE, int AHEAD>
__device__ __forceinline__ void rotate_token(const RopeParams& p, int t, int part, float2* turns) {
  const int lane = threadIdx.x & 31;
  NewTokens s;
  const int b = find_tokens(p, 0, s, [&](int, int, int to) { return to <= t; });
  if (b >= p.batch || t < s.q0) return;  // padding behind the last sequence
  const int pos = s.pos0 + (t - s.q0);
  if (pos < 0) return;
  const int page = CACHE ? page_at(p, b, pos) : -1;
  const int units = p.head_dim / kUnit;
  const bool fixed = 32 % units == 0;
  // steps: of 32 / units heads, or of one head (taken by as many lanes as it has units, in turns of 32)
  const int heads_a_step = fixed ? 32 / units : 1;
  const int steps_q = (p.heads_q + heads_a_step - 1) / heads_a_step, steps_kv = page >= 0 ? (p.heads_kv + heads_a_step - 1) / heads_a_step : 0;
  const int all = steps_q + 2 * steps_kv, per = (all + p.parts - 1) / p.parts;
  const int begin = part * per, end = min(begin + per, all);
  if (begin >= end) return;
  const int pairs = p.rotary / 2;
  for (int i = lane; i < pairs; i += 32) turns[i] = turn_of(p, pos, i);
  __syncwarp();
  const int64_t slot = page < 0 ? 0 : (int64_t)page * p.page_stride + (int64_t)(pos % p.page_size) * p.slot_stride;
  const int my_head = fixed ? lane / units : 0;
  for (int u = fixed ? lane % units : lane; u < units; u += 32) {  // (once where the unit is fixed)
    const Place at = place_of(p, u), plain{u * kUnit, u * kUnit + 4, false, false};
    float2 turn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) turn[i] = at.rotated ? turns[4 * u + i] : make_float2(1.f, 0.f);
    // the share of the steps [from, from + steps) of `heads` heads that is this part's: first step, and steps of this lane
    auto share = [&](int from, int steps, int heads, int& first) {
      first = max(begin - from, 0);
      const int last = min(end - from, steps);
      return min(last - first, (heads - my_head - first * heads_a_step + heads_a_step - 1) / heads_a_step);
    };
    int first;
    const int src_step = heads_a_step * p.head_dim;
    int n = share(0, steps_q, p.heads_q, first);
    if (n > 0) {
      const int head = first * heads_a_step + my_head;
      turn_units<true, AHEAD>(p.q + (int64_t)t * p.ld_q + head * p.head_dim, src_step, p.q_out + (int64_t)t * p.ld_q_out + head * p.head_dim, src_step, n, at, turn);
    }
    if (CACHE && page >= 0) {
      const int64_t dst_step = heads_a_step * p.head_stride;
      n = share(steps_q, steps_kv, p.heads_kv, first);
      int head = first * heads_a_step + my_head;
      if (n > 0)
        turn_units<true, AHEAD>(p.k_new + (int64_t)t * p.ld_new + head * p.head_dim, src_step, reinterpret_cast<__nv_bfloat16*>(p.k_cache) + slot + head * p.head_stride,
                                dst_step, n, at, turn);
      n = share(steps_q + steps_kv, steps_kv, p.heads_kv, first);
      head = first * heads_a_step + my_head;
      if (n > 0)
        turn_units<false, AHEAD>(p.v_new + (int64_t)t * p.ld_new + head * p.head_dim, src_step, reinterpret_cast<__nv_bfloat16*>(p.v_cache) + slot + head * p.head_stride,
                                 dst_step, n, plain, turn);
    }
  }
}

// Where the blocks of sequence b begin in the count of places for blocks: as many as its new tokens can touch, and no more
// than one and two halves of them, so that a place's sequence is found from cu_q alone.
__device__ __forceinline__ int64_t first_block_place(const RopeParams& p, int b, int from) {
  return (int64_t)(min(max(from, 0), p.tokens) >> p.scales.shift) + 2 * (int64_t)b;
}

// One block of one sequence, and some heads of K (KEYS) or of V of it.  A CTA.  FIXED: the units of a head divide 32, so that a lane has
// the same unit of every token it comes to.
template <pd_dtype T, bool KEYS, bool FIXED>
__device__ __forceinline__ void quantise_block(const RopeParams& p, int64_t place, int round, float2* turns, float* largest) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // the last sequence whose places begin at or in front of `place`
  NewTokens s;
  const int b = max(find_tokens(p, 1, s, [&](int i, int from, int) { return first_block_place(p, i, from) <= place; }) - 1, 0);
  const int shift = p.scales.shift;
  const int from = max(s.pos0, 0), to = s.pos0 + s.n;  // positions of the new tokens that have one
  if (from >= to) return;
  const int64_t index = (from >> shift) + (place - first_block_place(p, b, s.q0));
  if (index > ((to - 1) >> shift)) return;
  const int start = (int)index << shift;
  const int page = page_at(p, b, start);
  if (page < 0) return;
  const int first = max(start, from), last = (int)min((long long)start + (1ll << shift), (long long)to);
  const int old = first - start;  // older tokens of the block
  const int slot0 = start % p.page_size;

  const int heads_a_cta = kWarps / p.warps_a_head, part = warp % p.warps_a_head;
  const int rounds_k = p.rounds / 2;
  const int head = (KEYS ? round : round - rounds_k) * heads_a_cta + warp / p.warps_a_head;
  const bool mine = head < p.heads_kv;
  const int units = p.head_dim / kUnit;
  auto token_of = [&](int i) { return i / units; };  // of a unit in the warp's share
  const __nv_bfloat16* src = (KEYS ? p.k_new : p.v_new) + (int64_t)(s.q0 + first - s.pos0) * p.ld_new + (int64_t)head * p.head_dim;
  uint8_t* dst = (KEYS ? p.k_cache : p.v_cache) + (int64_t)page * p.page_stride + (int64_t)slot0 * p.slot_stride + (int64_t)head * p.head_stride;
  float* scale_at = (KEYS ? p.k_scale : p.v_scale) + p.scales.at(page, head, slot0);
  const float before = mine && old > 0 ? *scale_at : 0.f;

  const int per_warp = kGroup / units, per_group = per_warp * p.warps_a_head;  // tokens
  const int tokens = last - first, groups = (tokens + per_group - 1) / per_group;
  const int pairs = p.rotary / 2;
  auto place_in = [&](int u) {
    Place at = place_of(p, u);
    if (!KEYS) { at.rotated = at.split = false; at.first = u * kUnit; at.second = at.first + 4; }
    return at;
  };
  // unit j of this lane: its token in the warp's share, its unit of the head and its place in it
  const int my_token = lane / units, my_unit = lane % units, tokens_a_step = 32 / units;
  const Place my_place = place_in(my_unit);
  auto unit_j = [&](int j, int& t, int& u, Place& at) {
    if constexpr (FIXED) {
      t = my_token + j * tokens_a_step;
      u = my_unit;
      at = my_place;
    } else {
      t = token_of(lane + 32 * j);
      u = lane + 32 * j - t * units;
      at = place_in(u);
    }
  };
  // this warp's tokens of group g: from t0 of the block's new ones on, n units
  auto first_token = [&](int g) { return g * per_group + part * per_warp; };
  auto units_in = [&](int g) { return mine ? max(min(per_warp, tokens - first_token(g)), 0) * units : 0; };
  uint4 held[kHeld];
  auto load_group = [&](int g) {
    const int n = units_in(g);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = lane + 32 * j;
      if (i < n) {
        int t, u;
        Place at;
        unit_j(j, t, u, at);
        held[j] = load_unit(src + (int64_t)(first_token(g) + t) * p.ld_new, at);
      }
    }
  };
  auto turn_group = [&](int g) {  // cos and sin of the group's tokens; collective over the CTA
    if (!KEYS || pairs == 0) return;
    __syncthreads();
    const int n = min(per_group, tokens - g * per_group) * pairs;
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const int t = i / pairs;
      turns[i] = turn_of(p, first + g * per_group + t, i - t * pairs);
    }
    __syncthreads();
  };
  const float2* my_turns = turns + part * per_warp * pairs;
  float most = 0.f;
  uint32_t most2 = 0;
  for (int g = 0; g < groups; ++g) {
    load_group(g);
    turn_group(g);
    const int n = units_in(g);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = lane + 32 * j;
      if (i < n) {
        if constexpr (KEYS) {
          int t, u;
          Place at;
          unit_j(j, t, u, at);
          float x[8];
          rotate_unit(held[j], at, my_turns + t * pairs + 4 * u, x);
#pragma unroll
          for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(x[k]));
        } else {  // (bf16 magnitudes are in the order of their bits)
          const uint32_t w[4] = {held[j].x, held[j].y, held[j].z, held[j].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) most2 = __vmaxu2(most2, w[k] & 0x7fff7fffu);
        }
      }
    }
  }
  if constexpr (!KEYS) most = __uint_as_float(max(most2 << 16, most2 & 0xffff0000u));
  most = warp_max(most);
  if (p.warps_a_head > 1) {
    if (lane == 0) largest[warp] = most;
    __syncthreads();
    for (int k = 0; k < p.warps_a_head; ++k) most = fmaxf(most, largest[warp - part + k]);
  }
  // (a scale below the normal range would have no reciprocal)
  const float need = most > 0.f ? fmaxf(most / paged::q8_top<T>(), 1.17549435e-38f) : 0.f;
  const float scale = fmaxf(before, need);
  // x / scale, as x Q / m where the scale m / Q is new: keys and values are multiples of each other by small fractions often enough that
  // quotients lie on the border between two bytes, and m / Q rounded to fp32 would take them all to the same side of it.  One
  // refinement by the residual makes the product with the reciprocal as good as a division.
  const bool fresh = need >= before && most > 0x1p-100f && most < 0x1p100f;
  const float times = fresh ? paged::q8_top<T>() : 1.f, by = fresh ? most : scale, inv = by > 0.f ? 1.f / by : 0.f;
  auto quotient = [&](float x) {
    const float n = x * times, y = n * inv;
    return fmaf(fmaf(-y, by, n), inv, y);
  };
  for (int g = 0; g < groups; ++g) {
    if (groups > 1) {
      load_group(g);
      turn_group(g);
    }
    const int n = units_in(g);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = lane + 32 * j;
      if (i < n) {
        int t, u;
        Place at;
        unit_j(j, t, u, at);
        float x[8];
        rotate_unit(held[j], at, my_turns + t * pairs + 4 * u, x);
        uint32_t w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          w[k] = paged::q8_pair_from_float<T>(quotient(x[4 * k]), quotient(x[4 * k + 1])) |
                 paged::q8_pair_from_float<T>(quotient(x[4 * k + 2]), quotient(x[4 * k + 3])) << 16;
        uint8_t* row = dst + (int64_t)(old + first_token(g) + t) * p.slot_stride;
        if (at.split) {
          *reinterpret_cast<uint32_t*>(row + at.first) = w[0];
          *reinterpret_cast<uint32_t*>(row + at.second) = w[1];
        } else {
          *reinterpret_cast<uint2*>(row + at.first) = make_uint2(w[0], w[1]);
        }
      }
    }
  }
  if (!mine) return;
  if (old > 0 && scale > before) {
    // older values, to the larger step; the products in 64 bits, since 8 bits times the ratio of two scales can lie next to a border
    const double ratio = (double)before / (double)scale;
    constexpr int kAhead = 4;
    const int n = old * units, stride = 32 * p.warps_a_head;
    for (int i0 = part * 32 + lane; i0 < n; i0 += kAhead * stride) {
      uint2 v[kAhead];
      uint2* at[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const int i = min(i0 + a * stride, n - 1), t = token_of(i);
        at[a] = reinterpret_cast<uint2*>(dst + (int64_t)t * p.slot_stride + (i - t * units) * kUnit);
        v[a] = *at[a];
      }
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        if (i0 + a * stride >= n) break;
        uint32_t w[2] = {v[a].x, v[a].y};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float2 x = paged::q8_pair_to_float<T>(w[k]), y = paged::q8_pair_to_float<T>(w[k] >> 16);
          w[k] = paged::q8_pair_from_float<T>((float)(x.x * ratio), (float)(x.y * ratio)) |
                 paged::q8_pair_from_float<T>((float)(y.x * ratio), (float)(y.y * ratio)) << 16;
        }
        *at[a] = make_uint2(w[0], w[1]);
      }
    }
  }
  if (lane == 0 && part == 0) *scale_at = scale;
}

// bf16 cache: a warp for every part of a token.
__global__ void __launch_bounds__(kThreads) rope_kv_cache_append_kernel(const RopeParams p) {
  __shared__ float2 turns[kWarps][kMaxPairs];
  griddep_wait();
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5;
  const int64_t w = (int64_t)blockIdx.x * kWarps + warp;
  const int64_t t = w / p.parts;
  if (t < p.tokens) rotate_token<true, 4>(p, (int)t, (int)(w - t * p.parts), turns[warp]);
}

// 8-bit cache: the first CTAs take blocks of keys and values, the others parts of tokens' queries.
template <pd_dtype T>
__global__ void __launch_bounds__(kThreads, 4) rope_kv_cache_append_q8_kernel(const RopeParams p) {
  extern __shared__ float2 turns[];  // of a group's tokens: at most four pairs to a unit, kGroup units to each of warps_a_head warps
  __shared__ float largest[kWarps];
  static_assert(kWarps * kMaxPairs <= kGroup * 4);
  griddep_wait();
  griddep_launch_dependents();
  if ((int64_t)blockIdx.x < p.block_ctas) {
    const int round = blockIdx.x % p.rounds;
    const int64_t place = blockIdx.x / p.rounds;
    if (32 % (p.head_dim / kUnit) == 0) {
      if (round < p.rounds / 2) quantise_block<T, true, true>(p, place, round, turns, largest);
      else quantise_block<T, false, true>(p, place, round, turns, largest);
    } else {
      if (round < p.rounds / 2) quantise_block<T, true, false>(p, place, round, turns, largest);
      else quantise_block<T, false, false>(p, place, round, turns, largest);
    }
    return;
  }
  const int warp = threadIdx.x >> 5;
  const int64_t w = ((int64_t)blockIdx.x - p.block_ctas) * kWarps + warp;
  const int64_t t = w / p.parts;
  if (t < p.tokens) rotate_token<false, 4>(p, (int)t, (int)(w - t * p.parts), turns + warp * kMaxPairs);
}

}  // namespace
}  // namespace pd

extern "C" pd_status pd_rope_kv_cache_append(const pd_paged_attention_desc* desc, const pd_rope_desc* rope,
                                             const pd_cache_scales* scales, const void* q, void* q_out, const void* k_new,
                                             const void* v_new, int64_t ld_new, void* k_cache, void* v_cache,
                                             const int32_t* block_table, const int32_t* cu_q, const int32_t* kv_len,
                                             cudaStream_t stream) {
  using namespace pd;
  if (!desc || !rope) return PD_ERR_NULL_POINTER;
  const pd_paged_attention_desc& d = *desc;
  const bool queries = q != nullptr || q_out != nullptr;
  if (d.batch < 0 || d.tokens < 0 || d.heads_kv <= 0 || d.head_dim <= 0 || d.num_pages <= 0 || d.page_size <= 0 || d.max_pages <= 0 ||
      (queries && d.heads_q <= 0))
    return PD_ERR_BAD_SHAPE;
  if (rope->rotary_dim < 0 || rope->rotary_dim > d.head_dim || (rope->interleaved != 0 && rope->interleaved != 1) ||
      !(fabsf(rope->amplitude) <= 3.402823466e38f))
    return PD_ERR_BAD_SHAPE;
  if (scales && (!paged::q8_dtype(scales->dtype) || !paged::q8_block_valid(scales->block, d.page_size))) return PD_ERR_BAD_SHAPE;
  if (d.head_dim % kUnit != 0 || d.head_dim > kMaxDim || rope->rotary_dim % 8 != 0 || d.heads_kv > 65536 || d.batch > 65535 ||
      d.tokens > kMaxIndex || (queries && d.heads_q > 65536))
    return PD_ERR_UNSUPPORTED;
  if (ld_new < (int64_t)d.heads_kv * d.head_dim || d.page_stride <= 0 || d.slot_stride <= 0 || d.head_stride <= 0) return PD_ERR_BAD_SHAPE;
  if (queries && (d.ld_q < (int64_t)d.heads_q * d.head_dim || d.ld_out < (int64_t)d.heads_q * d.head_dim)) return PD_ERR_BAD_SHAPE;
  if (d.batch == 0 || d.tokens == 0) return PD_OK;
  if (!k_new || !v_new || !k_cache || !v_cache || !block_table || !cu_q || !kv_len || (queries && (!q || !q_out)) ||
      (rope->rotary_dim > 0 && !rope->inv_freq) || (scales && (!scales->k_scale || !scales->v_scale)))
    return PD_ERR_NULL_POINTER;
  auto bits = [](const void* v) { return reinterpret_cast<uintptr_t>(v); };
  const int64_t cache_strides = d.page_stride | d.slot_stride | d.head_stride;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(q) || !aligned16(q_out) ||
      (ld_new & 7) != 0 || (queries && ((d.ld_q | d.ld_out) & 7) != 0) || (cache_strides & (scales ? 15 : 7)) != 0 ||
      ((bits(block_table) | bits(cu_q) | bits(kv_len) | bits(rope->inv_freq)) & 3u) != 0 ||
      (scales && ((bits(scales->k_scale) | bits(scales->v_scale)) & 3u) != 0))
    return PD_ERR_ALIGNMENT;

  RopeParams p{};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.k_new = static_cast<const __nv_bfloat16*>(k_new);
  p.v_new = static_cast<const __nv_bfloat16*>(v_new);
  p.k_cache = static_cast<uint8_t*>(k_cache);
  p.v_cache = static_cast<uint8_t*>(v_cache);
  p.inv_freq = rope->inv_freq;
  p.block_table = block_table; p.cu_q = cu_q; p.kv_len = kv_len;
  p.ld_q = d.ld_q; p.ld_q_out = d.ld_out; p.ld_new = ld_new;
  p.page_stride = d.page_stride; p.slot_stride = d.slot_stride; p.head_stride = d.head_stride;
  p.amplitude = rope->amplitude; p.rotary = rope->rotary_dim; p.interleaved = rope->interleaved;
  p.batch = d.batch; p.tokens = d.tokens; p.heads_q = queries ? d.heads_q : 0; p.heads_kv = d.heads_kv; p.head_dim = d.head_dim;
  p.num_pages = d.num_pages; p.page_size = d.page_size; p.max_pages = d.max_pages;
  // A warp per token while tokens fill the SMs (eight warps each), several for fewer tokens, none with less than 64 units.
  const int64_t units = ((int64_t)p.heads_q + (scales ? 0 : 2 * (int64_t)d.heads_kv)) * (d.head_dim / kUnit);
  int64_t parts = (148 * kWarps + d.tokens - 1) / d.tokens;
  if (parts > (units + 63) / 64) parts = (units + 63) / 64;
  p.parts = (int)(parts < 1 ? 1 : parts);
  const int64_t token_ctas = units == 0 ? 0 : ((int64_t)d.tokens * p.parts + kWarps - 1) / kWarps;
  if (scales) {
    p.scales = paged::make_scales(*scales, d.heads_kv, d.page_size);
    p.k_scale = scales->k_scale; p.v_scale = scales->v_scale;
    // as many warps to a head as hold a whole block's units between the two passes (by the block alone: with few heads and short blocks, or
    // few new tokens in long ones, some of a CTA's warps have nothing to do)
    p.warps_a_head = 1;
    while (p.warps_a_head < kWarps && (int64_t)scales->block * (d.head_dim / kUnit) > (int64_t)kGroup * p.warps_a_head) p.warps_a_head *= 2;
    const int heads_a_cta = kWarps / p.warps_a_head;
    p.rounds = 2 * ((d.heads_kv + heads_a_cta - 1) / heads_a_cta);
    p.block_ctas = (((int64_t)d.tokens >> p.scales.shift) + 2 * (int64_t)d.batch) * p.rounds;
  }
  const int64_t ctas = p.block_ctas + token_ctas;
  if (ctas > 0x7fffffff) return PD_ERR_UNSUPPORTED;
  if (pd_status st = require_sm100(); st != PD_OK) return st;
  logf("rope kv cache append: %d tokens of %d sequences, %s cache, %lld + %lld CTAs", d.tokens, d.batch,
       !scales ? "bf16" : scales->dtype == PD_I8 ? "int8" : "e4m3", (long long)p.block_ctas, (long long)token_ctas);
  const dim3 grid((unsigned)ctas), block(kThreads);
  if (!scales) {
    launch_pdl(rope_kv_cache_append_kernel, grid, block, 0, stream, p);
    return check_launch();
  }
  auto kernel = scales->dtype == PD_I8 ? rope_kv_cache_append_q8_kernel<PD_I8> : rope_kv_cache_append_q8_kernel<PD_E4M3>;
  static PerDeviceFlag smem_allowed[2];
  const size_t turn_bytes = (size_t)p.warps_a_head * kGroup * 4 * sizeof(float2);
  if (pd_status st = allow_dynamic_smem(kernel, kWarps * kGroup * 4 * (int)sizeof(float2), smem_allowed[scales->dtype == PD_I8]); st != PD_OK) return st;
  launch_pdl(kernel, grid, block, turn_bytes, stream, p);
  return check_launch();
}
