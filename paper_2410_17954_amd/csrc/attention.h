// What the attention kernels over packed prompts and over a cache in 4 bits share:
// tiles of S^T = K Q^T and O^T = V^T P^T on 16x16 MFMAs, where lane (r, q4) = (lane %
// 16, lane / 16) holds scores of query r for keys 4 q4 .. 4 q4 + 3, the running
// softmax over them, and the join of key ranges that blocks took.
#pragma once

#include "common.h"

#include <math.h>

namespace moe {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float quad_max(float v) {   // over the four lanes of a query
  v = fmaxf(v, __shfl_xor(v, 16, kWave));
  return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// Scores -> softmax numerators 2^(s scale2 - m) in place, for MT tiles of queries and
// KT tiles of keys. m: their reference, kSlack above the largest score when it was
// raised, and raised again (l and o rescaled) only where a score exceeds it, so that
// most steps rescale nothing. Numerators are at most 1 (but for the rounding of m): a
// value times one is finite if the value is. One branch for all tiles. Next to a
// reference kSlack away a difference is rounded to 2^-21 of 8: little beside numerators
// of bf16; float32 ones have 2^-22 of 4, where rescaling costs 1 % of small calls (300
// tokens of 8 heads of 64: 14.9 -> 15.0 us, without slack 15.4).
template <typename Tv>
constexpr float kSlack = sizeof(Tv) == 2 ? 8.f : 4.f;

template <typename Tv, int MT, int KT, int DT>
__device__ __forceinline__ void softmax_step(f32x4_t (&s)[MT][KT], float (&m)[MT], float (&l)[MT],
                                             f32x4_t (&o)[MT][DT], float scale2) {
  float mx[MT];
  bool raise = false;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    mx[i] = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx[i] = fmaxf(mx[i], s[i][kt][e]);
    raise = raise | (mx[i] * scale2 > m[i]);
  }
  if (ballot(raise)) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      mx[i] = quad_max(mx[i]) * scale2;
      const float to = mx[i] > m[i] ? mx[i] + kSlack<Tv> : m[i];
      const float f = to == m[i] ? 1.f : __builtin_amdgcn_exp2f(m[i] - to);   // 0 from -inf
      m[i] = to;
      l[i] *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[i][dt] *= f;
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const float mu = m[i] == -INFINITY ? 0.f : m[i];         // nothing but -inf so far
    float sum = 0.f;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[i][kt][e], scale2, -mu));
        s[i][kt][e] = p;
        sum += p;
      }
    l[i] += sum;
  }
}

// Four values of a row's result, the row on 16 bytes.
__device__ __forceinline__ void put4(uint16_t* dst, f32x4_t o) {
  const uint32_t lo = (uint32_t)f32_to_bf16(o[0]) | (uint32_t)f32_to_bf16(o[1]) << 16;
  const uint32_t hi = (uint32_t)f32_to_bf16(o[2]) | (uint32_t)f32_to_bf16(o[3]) << 16;
  *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
}
__device__ __forceinline__ void put4(float* dst, f32x4_t o) { *reinterpret_cast<f32x4_t*>(dst) = o; }
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// scale as kernels take it: never 0, which would make a masked key's score NaN; then
// q & keep ^ flip has no bits, and its signs are turned where scale is negative.
struct ScoreScale { float scale2; uint32_t keep, flip; };
inline ScoreScale score_scale(float scale, bool bf16) {
  const bool none = fabsf(scale) < 1e-37f;
  return {none ? 1.f : fabsf(scale) * kLog2e, none ? 0u : ~0u,
          none || scale >= 0.f ? 0u : bf16 ? 0x80008000u : 0x80000000u};
}

// ---------------------------------------------------------------- join
// part_o [splits][RH][D], part_ml [splits][RH] (reference in log2, sum; sum 0: o is not
// read; of a reference of -inf any other sum adds 0, o only what is no number) -> out [RH, D], lse [RH] of the rows offsets[0] .. offsets[n_off - 1] - 1 (RH /
// heads rows; all without offsets).
struct JoinArgs {
  const float* part_o;
  const float2* part_ml;
  const int32_t* offsets;
  int64_t n_off, RH;
  int heads, D, splits;
  void* out;
  float* lse;
};

constexpr int kJoinThreads = 256, kJoinBlocks = 512;
// Few rows have their dimensions cut over blocks, 32 of them at least, until there are this
// many (32 rows and heads of 128, 256 splits: call 37.3 -> 35.4 us; eight of 256 behind
// 30000 keys 17.1 -> 14.6; blocks of 1024 threads, whole rows each, were the former).
constexpr int kJoinDimBlocks = 256;

namespace {                                      // a kernel of its own for every source

// tpr threads of a block (8 to 64) take four dimensions each of a row and head, those
// from blockIdx.y on, and sg groups of them share the splits (a power of two; groups are
// added up in a tree: a fixed order). A thread's loads do not wait for each other: the
// maximum over all splits comes first.
template <typename Tv>
__global__ void __launch_bounds__(kJoinThreads)
attention_join_kernel(JoinArgs a, int tpr_shift, int sg_shift) {
  constexpr int T = kJoinThreads;
  __shared__ f32x4_t s_o[T];
  __shared__ float s_l[T];
  const int tpr = 1 << tpr_shift, sg = 1 << sg_shift;
  const int64_t at = (int64_t)blockIdx.x * (T >> (tpr_shift + sg_shift)) +
                     (threadIdx.x >> (tpr_shift + sg_shift));
  const int x = threadIdx.x & (tpr - 1), d = 4 * ((int)blockIdx.y * tpr + x);
  const int g = (threadIdx.x >> tpr_shift) & (sg - 1);
  const int64_t row = at / a.heads;
  bool live = at < a.RH;
  if (a.offsets) live = live && row >= a.offsets[0] && row < a.offsets[a.n_off - 1];
  const bool mine = live && d < a.D;
  float m = -INFINITY;
  auto lanes_max = [&]() {
    for (int n = tpr >> 1; n > 0; n >>= 1) m = fmaxf(m, __shfl_xor(m, n, kWave));
  };
  if (live)
    for (int p = g * tpr + x; p < a.splits; p += sg * tpr) m = fmaxf(m, a.part_ml[p * a.RH + at].x);
  lanes_max();
  if (sg > 1) {
    const int first = (threadIdx.x >> (tpr_shift + sg_shift)) << sg_shift;
    if (x == 0) s_l[first + g] = m;
    __syncthreads();
    for (int i = x; i < sg; i += tpr) m = fmaxf(m, s_l[first + i]);
    lanes_max();
    __syncthreads();                             // s_l is rewritten below
  }
  const float mu = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  if (mine) {
#pragma unroll 4
    for (int p = g; p < a.splits; p += sg) {
      const float2 ml = a.part_ml[p * a.RH + at];
      f32x4_t po = *reinterpret_cast<const f32x4_t*>(a.part_o + (p * a.RH + at) * a.D + d);
      float f = __builtin_amdgcn_exp2f(ml.x - mu);
      if (ml.y == 0.f) {                         // a split without keys wrote no O
        f = 0.f;
        po = f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
      l = fmaf(ml.y, f, l);
#pragma unroll
      for (int e = 0; e < 4; ++e)                // an infinity counts whatever its weight
        o[e] = fmaf(po[e], fabsf(po[e]) == INFINITY ? 1.f : f, o[e]);
    }
  }
  for (int n = sg >> 1; n > 0; n >>= 1) {
    s_o[threadIdx.x] = o;
    s_l[threadIdx.x] = l;
    __syncthreads();
    if (g < n) {
      o += s_o[threadIdx.x + (n << tpr_shift)];
      l += s_l[threadIdx.x + (n << tpr_shift)];
    }
    __syncthreads();
  }
  if (g != 0 || !mine) return;
  if (l == 0.f) o = f32x4_t{0.f, 0.f, 0.f, 0.f};
  else o *= 1.f / l;
  put4(static_cast<Tv*>(a.out) + at * a.D + d, o);
  if (a.lse && d == 0) a.lse[at] = lse_of(m, l);
}

template <typename Tv>
int attention_join(const JoinArgs& a, hipStream_t st) {
  constexpr int t_shift = 8;
  static_assert(kJoinThreads == 1 << t_shift, "threads of a block");
  int tpr_shift = a.D <= 64 ? 4 : a.D <= 128 ? 5 : 6, sg_shift = 0;
  while (tpr_shift > 3 && a.RH * ceil_div(a.D, 4 << tpr_shift) < kJoinDimBlocks) --tpr_shift;
  const int64_t dims = ceil_div(a.D, 4 << tpr_shift);
  // groups until the card has blocks enough: with many rows threads take all splits
  auto blocks = [&]() { return ceil_div(a.RH, kJoinThreads >> (tpr_shift + sg_shift)); };
  while (sg_shift < t_shift - tpr_shift && (2 << sg_shift) <= a.splits &&
         blocks() * dims < kJoinBlocks)
    ++sg_shift;
  attention_join_kernel<Tv><<<dim3((unsigned)blocks(), (unsigned)dims), dim3(kJoinThreads), 0, st>>>(
      a, tpr_shift, sg_shift);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

}  // namespace

}  // namespace moe
