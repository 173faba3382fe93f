// moe_token_logprobs: log-probabilities of given tokens, entropy, best alternatives.
//
// Bound by reading the logits once. A block takes a row, its threads 16 bytes at a time
// in turn, the next ones in flight, and each keeps a reference ref, s = sum e^(z - ref)
// and h = sum e^(z - ref) (z - ref) of what it saw:
//   ln sum e^z = M + ln S,   entropy = ln S - H / S
// with S and H the threads' sums brought to the best logit M. A reference is
// raised only where a logit exceeds it by more than kSlack, so almost never after the
// first ones. Exponentials and short sums are of float32: S is off by up to 2^-17 of
// itself. Where S is below 2 that is much beside ln S, which is next to 0: the threads
// that hold the best logit then have their logits read again and the others' terms summed
// apart from it, S = C + rest with C the (one or two) terms that are 1. So what is next to
// 0 is off by a part of itself, and with one token left 0. Such a row takes 1 us more (1 x
// 32000 float32 8.3 -> 9.2, 2000 x 128000 97.5 -> 99); to count the best while any row is
// read took 2 of 8.3 and 13 of 104.
// Best alternatives need no second pass over the row: of kGroups groups of threads the
// n-th largest of their maxima, cut to some leading bits, is a bound T that n logits
// reach, and only threads whose own maximum reaches T hold more of them, about n. A
// wave reads such a thread's logits again, a lane each 16 bytes, and those from T on
// are ranked by counting.
#include "moeflow_prompt.h"
#include "common.h"
#include "rows.h"
#include "spans.h"

#include <float.h>
#include <math.h>

#include <algorithm>

namespace moe {
namespace {

constexpr int kMaxTop = 64;
constexpr int kGroups = 256;
constexpr int kKeys = 1024;                      // logits from T on that are ranked
constexpr int kBoundBits = 20;
constexpr float kSlack = 8.f;
constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes from an address that is only element-aligned.
struct __attribute__((packed, aligned(2))) Bytes16 { uint32_t w[4]; };
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));

template <typename Tv> struct LpVec;
template <> struct LpVec<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const Bytes16& b, float* out) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      out[2 * i] = __uint_as_float(b.w[i] << 16);
      out[2 * i + 1] = __uint_as_float(b.w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float one(const uint16_t* p) { return bf16_to_f32(*p); }
};
template <> struct LpVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const Bytes16& b, float* out) {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = __uint_as_float(b.w[i]);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};

struct LpArgs {
  const void* logits;
  int64_t V, stride, m;
  const int32_t* tokens;
  int n_top;
  float *logprobs, *entropy;
  int32_t* top_tokens;
  float* top_logprobs;
};

// Sums of one thread (or wave, or block): float32 over up to 32 logits, then float64.
struct LpSum {
  float ref;
  double s, h;
};

// e^d, d <= 0: the power of two in whole steps apart from the float32 exponential of the
// rest, so that it is off by an ulp of float32 however small it is; 0 far below.
__device__ __forceinline__ double lp_exp(double d) {
  const double x = fmax(d * 1.4426950408889634, -1100.0), n = rint(x);
  return ldexp((double)__builtin_amdgcn_exp2f((float)(x - n)), (int)n);
}

// ln(1 + x), x >= 0, off by 2^-33 of itself: with 1 + x = 2^e (1 + f), 1 + f within a
// factor sqrt(2) of 1 (f = x where e is 0, however small), ln(1 + f) = 2 artanh(f / (2 + f))
// by its series. NaN of NaN.
__device__ __forceinline__ double lp_log1p(double x) {
  int e;
  double m = frexp(1.0 + x, &e);
  if (m < 0.7071067811865476) {
    m *= 2.0;
    --e;
  }
  const double f = e == 0 ? x : m - 1.0, y = 2.0 + f;
  double c = __builtin_amdgcn_rcp(y);            // and a step of Newton's
  c = fma(c, fma(-y, c, 1.0), c);
  const double r = f * c, z = r * r;
  double p = fma(z, 1.0 / 11, 1.0 / 9);
  p = fma(z, p, 1.0 / 7);
  p = fma(z, p, 1.0 / 5);
  p = fma(z, p, 1.0 / 3);
  return fma((double)e, 0.6931471805599453, 2.0 * fma(r * z, p, r));
}

// Brings sums to a reference at least as large. No logits: ref -inf, sums 0.
__device__ __forceinline__ void lp_raise(LpSum& x, float to) {
  if (x.ref != to && x.ref != -INFINITY) {
    const double d = (double)x.ref - (double)to, f = lp_exp(d);
    // a factor that underflows leaves nothing, whatever the difference
    x.h = f > 0.0 || x.s != x.s ? f * (x.h + d * x.s) : 0.0;
    x.s *= f;
  }
  x.ref = to;
}

// Over the wave: rows of 16 lanes by DPP, then the four rows.
__device__ __forceinline__ double lp_lane(double v, int l) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, l);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), l);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
template <typename T>
__device__ __forceinline__ T lp_row_sum(T v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  return v + dpp<0x140>(v);
}
__device__ __forceinline__ double lp_wave_sum(double v) {
  v = lp_row_sum(v);
  return (lp_lane(v, 0) + lp_lane(v, 16)) + (lp_lane(v, 32) + lp_lane(v, 48));
}
__device__ __forceinline__ float lp_row_max(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  return fmaxf(v, dpp<0x140>(v));
}
__device__ __forceinline__ float lp_wave_max(float v) {
  v = lp_row_max(v);
  auto at = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return fmaxf(fmaxf(at(0), at(16)), fmaxf(at(32), at(48)));
}

// T threads, U 16-byte loads of each in flight beside the ones in work.
template <typename Tv, int T, int U, bool NT>
__global__ void __launch_bounds__(T)
lp_kernel(LpArgs a) {
  using LV = LpVec<Tv>;
  constexpr int VE = LV::N, W = T / kWave;
  static_assert(U * VE % 32 == 0 || 32 % (U * VE) == 0, "float32 sums of at most 32 logits");
  constexpr int PART = U * VE < 32 ? U * VE : 32;
  __shared__ float s_ref[W];
  __shared__ double s_s[W], s_h[W];
  __shared__ int s_ones[W];
  __shared__ float s_max[kGroups];
  __shared__ int s_count;
  __shared__ float s_key[kKeys];
  __shared__ int32_t s_idx[kKeys];
  const int64_t row = blockIdx.x;
  const Tv* const z = static_cast<const Tv*>(a.logits) + row * a.stride;
  const int t = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int V = (int)a.V, nvec = V / VE, rest = V - nvec * VE;

  Bytes16 raw[U];
  auto load = [&](int at) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at + u * T < nvec) {
        const Bytes16* const from = reinterpret_cast<const Bytes16*>(z + (int64_t)(at + u * T) * VE);
        if constexpr (NT) raw[u] = __builtin_bit_cast(Bytes16, __builtin_nontemporal_load(
            reinterpret_cast<const u32x4_any_t*>(from)));
        else raw[u] = *from;
      }
  };
  load(t);
  // given tokens: their logits are on the way while the row is
  int32_t tok = -1;
  float ztok = 0.f;
  if (t < a.m) {
    tok = a.tokens[row * a.m + t];
    if (tok >= 0 && tok < V) ztok = LV::one(z + tok);
  }
  if (t == 0) s_count = 0;

  LpSum x = {-INFINITY, 0.0, 0.0};
  float best = -INFINITY;                        // a NaN is no maximum
  auto add = [&](const float* v, int n) {
    float top = v[0];
#pragma unroll
    for (int i = 1; i < n; ++i) top = fmaxf(top, v[i]);
    best = fmaxf(best, top);
    if (top > x.ref + kSlack) lp_raise(x, top);
    const float mu = x.ref == -INFINITY ? 0.f : x.ref;       // nothing but -inf so far
    float s = 0.f, h = 0.f;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float d = v[i] - mu, e = __builtin_amdgcn_exp2f(d * kLog2e);
      s += e;
      h = fmaf(e, fmaxf(d, -200.f), h);          // 0 times -inf is 0 here; NaN stays in e
    }
    x.s += (double)s;
    x.h += (double)h;
  };
  for (int at = t; at < nvec; at += U * T) {
    float v[U * VE];
#pragma unroll
    for (int u = 0; u < U; ++u) LV::unpack(raw[u], v + u * VE);
    const bool whole = at + (U - 1) * T < nvec;
    if (!whole) {
#pragma unroll
      for (int u = 1; u < U; ++u)
        if (at + u * T >= nvec)
#pragma unroll
          for (int i = 0; i < VE; ++i) v[u * VE + i] = -INFINITY;
    }
    if (at + U * T < nvec) load(at + U * T);
#pragma unroll
    for (int i = 0; i < U * VE; i += PART) add(v + i, PART);
  }
  if (t < rest) {
    const float v = LV::one(z + nvec * VE + t);
    add(&v, 1);
  }

  // the waves' sums and the groups' maxima
  const float ref = lp_wave_max(best);
  lp_raise(x, ref);
  auto publish = [&](double s, double h) {
    s = lp_wave_sum(s);
    h = lp_wave_sum(h);
    if (lane == 0) {
      s_s[wave] = s;
      s_h[wave] = h;
    }
  };
  if (lane == 0) s_ref[wave] = ref;
  publish(x.s, x.h);
  float gmax = best;                             // a group is T / kGroups neighbours
  if (T > kGroups) gmax = fmaxf(gmax, dpp<0xB1>(gmax));
  if (T > 2 * kGroups) gmax = fmaxf(gmax, dpp<0x4E>(gmax));
  if (t % (T / kGroups) == 0) s_max[t / (T / kGroups)] = gmax;
  __syncthreads();

  // the row's: every wave for itself, lane w % 16 the sums of wave w
  const int of = lane % 16 % W;
  const bool one = lane % 16 < W;
  const float w_ref = s_ref[of];
  float M = lp_row_max(w_ref);
  const double w_d = w_ref == M ? 0.0 : (double)w_ref - (double)M;
  const double w_f = one ? lp_exp(w_d) : 0.0;    // 0 far below: whatever the difference
  double S, H;
  auto sum_waves = [&]() {
    const double s = s_s[of], h = s_h[of];
    const bool some = w_f > 0.0 || s != s;
    S = lp_row_sum(w_f * s);
    H = lp_row_sum(some ? w_f * (h + w_d * s) : 0.0);
  };
  sum_waves();
  const bool none = M == -INFINITY && S == 0.0;
  double lnS = 0.0;
  if (!(S < 2.0)) {
    lnS = lp_log1p(S - 1.0);                     // NaN of a row with a NaN or +inf
  } else if (!none) {                            // the same in every wave
    __syncthreads();                             // s_s and s_h are rewritten below
    int ones = 0;
    const uint64_t owners = ballot(best == M);
    if (owners) {                                // this wave's reference is M
      double s = best == M ? 0.0 : x.s, h = best == M ? 0.0 : x.h;
      auto others = [&](const float* v, int n) {
        float s32 = 0.f, h32 = 0.f;
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const float d = v[i] - M;
          const float e = v[i] == M ? 0.f : __builtin_amdgcn_exp2f(d * kLog2e);
          ones += v[i] == M;
          s32 += e;
          h32 = fmaf(e, fmaxf(d, -200.f), h32);
        }
        s += (double)s32;
        h += (double)h32;
      };
#pragma unroll 1
      for (uint64_t own = owners; own; own &= own - 1) {
        const int o = wave * kWave + __ffsll((unsigned long long)own) - 1;
#pragma unroll 1
        for (int at = o + lane * T; at < nvec; at += kWave * T) {
          float v[VE];
          LV::unpack(*reinterpret_cast<const Bytes16*>(z + (int64_t)at * VE), v);
          others(v, VE);
        }
        if (lane == 0 && o < rest) {
          const float v = LV::one(z + nvec * VE + o);
          others(&v, 1);
        }
      }
      publish(s, h);
      ones = (int)lp_wave_sum((double)ones);
    }
    if (lane == 0) s_ones[wave] = ones;
    __syncthreads();
    sum_waves();
    const int C = lp_row_sum(one ? s_ones[of] : 0);
    lnS = lp_log1p((double)(C - 1) + S);
    S += (double)C;
  }
  if (none) M = 0.f;
  if (t == 0 && a.entropy) a.entropy[row] = none ? 0.f : (float)(lnS - H / S);
  // the difference to the maximum first: beside a mask's lowest number ln S is lost
  auto logprob = [&](float v) { return (float)((double)v - (double)M - lnS); };
  for (int64_t j = t; j < a.m; j += T) {
    if (j >= T) {
      tok = a.tokens[row * a.m + j];
      ztok = tok >= 0 && tok < V ? LV::one(z + tok) : 0.f;
    }
    a.logprobs[row * a.m + j] = tok >= 0 && tok < V ? logprob(ztok) : -INFINITY;
  }
  if (a.n_top == 0) return;
  int32_t* const out_idx = a.top_tokens + row * a.n_top;
  float* const out_val = a.top_logprobs + row * a.n_top;
  if (lnS != lnS) {
    for (int j = t; j < a.n_top; j += T) {
      out_idx[j] = -1;
      out_val[j] = -INFINITY;
    }
    return;
  }
  // T: the largest number of kBoundBits leading bits that n_top groups reach, bit by bit
  // over the maxima's order; not below the lowest number, -inf is no candidate
  uint32_t key[kGroups / kWave], bound = 0;
#pragma unroll
  for (int i = 0; i < kGroups / kWave; ++i) key[i] = float_order(s_max[i * kWave + lane]);
  for (int bit = 31; bit > 31 - kBoundBits; --bit) {
    const uint32_t to = bound | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < kGroups / kWave; ++i) n += (int)__popcll(ballot(key[i] >= to));
    if (n >= a.n_top) bound = to;
  }
  bound = max(bound, float_order(-FLT_MAX));
  auto offer = [&](float v, int i) {
    const int at = atomicAdd(&s_count, 1);
    if (at < kKeys) {
      s_key[at] = v;
      s_idx[at] = i;
    }
  };
  // a wave reads again what its threads of a maximum from T on had read
  for (uint64_t own = ballot(float_order(best) >= bound); own; own &= own - 1) {
    // too many already: the passes below take over
    if (__builtin_amdgcn_readfirstlane(*static_cast<volatile int*>(&s_count)) > kKeys) break;
    const int o = wave * kWave + __ffsll((unsigned long long)own) - 1;
    for (int at = o + lane * T; at < nvec; at += kWave * T) {
      float v[VE];
      LV::unpack(*reinterpret_cast<const Bytes16*>(z + (int64_t)at * VE), v);
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (float_order(v[i]) >= bound) offer(v[i], at * VE + i);
    }
    if (lane == 0 && o < rest) {
      const float v = LV::one(z + nvec * VE + o);
      if (float_order(v) >= bound) offer(v, nvec * VE + o);
    }
  }
  __syncthreads();
  int count = s_count;
  if (count > kKeys) {
    // That many equal ones at the bound (a mask of the lowest number that leaves fewer
    // than n_top): the n_top-th largest exactly, eight bits of its order at a time from
    // how often each continuation of them occurs, then what is above it and the first
    // of its equals (64 rows of 128000, three left, 20 places: 105 us; one pass over the
    // row a place took 708).
    int32_t* const often = s_idx;                // of the 256 continuations
    const uint32_t low = float_order(-FLT_MAX);
    uint32_t nth = 0, bits = 0;
    int left = a.n_top;                          // equals of nth, in the bits so far, to take
    auto some = [&](float (&v)[4], int i) {      // loads that do not wait for each other
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = i + u * T < V ? LV::one(z + i + u * T) : -INFINITY;
    };
    for (int shift = 24; shift >= (VE == 8 ? 16 : 0); shift -= 8) {   // bf16: the rest is its sign
      __syncthreads();
      for (int i = t; i < 256; i += T) often[i] = 0;
      __syncthreads();
      for (int i0 = t; i0 - t < V; i0 += 4 * T) {
        float v[4];
        some(v, i0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t k = float_order(v[u]);
          const bool in = k >= low && (k & bits) == nth;
          const int next = (int)(k >> shift & 255u);
          if (const uint64_t any = ballot(in)) { // the first lane's and its equals at once
            const int first = __ffsll((unsigned long long)any) - 1;
            const bool same = in && next == __builtin_amdgcn_readlane(next, first);
            const uint64_t equals = ballot(same);
            if (lane == first) atomicAdd(often + next, (int)__popcll(equals));
            else if (in && !same) atomicAdd(often + next, 1);
          }
        }
      }
      __syncthreads();
      // every wave for itself, lane l the continuations 4 l .. 4 l + 3
      int c[4], mine = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) mine += c[e] = often[4 * lane + e];
      int from = mine;                           // as often from the lane's on
      for (int d = 1; d < kWave; d <<= 1) {
        const int more = __shfl_down(from, d, kWave);
        if (lane + d < kWave) from += more;
      }
      const int l = 63 - __clzll((long long)ballot(from >= left));
      left -= __builtin_amdgcn_readlane(from - mine, l);
      int next = 4 * l + 3;
#pragma unroll
      for (int e = 3; e > 0; --e) {
        const int n = __builtin_amdgcn_readlane(c[e], l);
        if (next == 4 * l + e && left > n) {
          left -= n;
          --next;
        }
      }
      nth |= (uint32_t)next << shift;
      bits |= 255u << shift;
    }
    __syncthreads();                             // s_idx and s_count are rewritten below
    if (t == 0) s_count = 0;
    __syncthreads();
    for (int i = t; i < V; i += 4 * T) {
      float v[4];
      some(v, i);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if ((float_order(v[u]) & bits) > nth) offer(v[u], i + u * T);
    }
    __shared__ int s_equals[W];
    for (int i0 = 0; i0 < V && left > 0; i0 += T) {
      const int i = i0 + t;
      const float v = i < V ? LV::one(z + i) : -INFINITY;
      const bool in = (float_order(v) & bits) == nth;
      const uint64_t equals = ballot(in);
      if (lane == 0) s_equals[wave] = (int)__popcll(equals);
      __syncthreads();
      int before = (int)__popcll(equals & ((1ull << lane) - 1)), all = 0;
      for (int w = 0; w < W; ++w) {
        if (w < wave) before += s_equals[w];
        all += s_equals[w];
      }
      if (in && before < left) offer(v, i);
      left -= all;
      __syncthreads();                           // s_equals is rewritten next
    }
    __syncthreads();
    count = s_count;                             // n_top
  }
  for (int i = t; i < count; i += T) {
    const float v = s_key[i];
    const int32_t id = s_idx[i];
    int r = 0;
#pragma unroll 4
    for (int o = 0; o < count; ++o)
      r += (s_key[o] > v) | ((s_key[o] == v) & (s_idx[o] < id));
    if (r < a.n_top) {
      out_idx[r] = id;
      out_val[r] = logprob(v);
    }
  }
  for (int j = count + t; j < a.n_top; j += T) {
    out_idx[j] = -1;
    out_val[j] = -INFINITY;
  }
}

bool lp_ok(int64_t R, int64_t V, int64_t m, int32_t n_top) {
  return R >= 1 && V >= 1 && m >= 0 && n_top >= 0;
}
bool lp_supported(int64_t R, int64_t V, int64_t m, int32_t n_top) {
  return n_top <= kMaxTop && V <= (1 << 24) && R < (1 << 22) && m < ((int64_t)1 << 31) / R;
}

// Rows that the compute units hold at once go to blocks of 1024 threads, which have more
// of a row in flight (one row of 128000 bf16 logits 11 us without alternatives, with 256
// threads 29); more rows to blocks of 256, eight a compute unit (300 rows of 32000: 8.2
// us, of 1024 threads 13.7), whose logits are more than the caches keep, so that the
// non-temporal hint pays (2000 rows of 128000: 97 us, 5.3 TB/s, without it 106; 64 rows,
// which the caches hold, 13.4 with it, 11.6 without).
template <typename Tv>
int lp_run(const LpArgs& a, int64_t R, hipStream_t st) {
  if (R <= 256) lp_kernel<Tv, 1024, 8, false><<<dim3((unsigned)R), dim3(1024), 0, st>>>(a);
  else lp_kernel<Tv, 256, 4, true><<<dim3((unsigned)R), dim3(256), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_token_logprobs_workspace(int64_t R, int64_t V, int64_t m, int32_t n_top) {
  return 0;
}

extern "C" int moe_token_logprobs(const void* logits, int32_t dtype, int64_t R, int64_t V,
                                  int64_t stride, const int32_t* tokens, int64_t m, int32_t n_top,
                                  float* logprobs, float* entropy, int32_t* top_tokens,
                                  float* top_logprobs, void* workspace, size_t ws_bytes,
                                  void* stream) {
  using namespace moe;
  MOE_CHECK_ARG(logits && valid_dtype(dtype) && lp_ok(R, V, m, n_top) && stride >= V);
  MOE_CHECK_ARG(m == 0 || (tokens && logprobs));
  MOE_CHECK_ARG(n_top == 0 || (top_tokens && top_logprobs));
  MOE_CHECK_ARG(m > 0 || n_top > 0 || entropy);
  const int64_t elt = dtype == MOE_BF16 ? 2 : 4;
  MOE_CHECK_ARG(reinterpret_cast<uintptr_t>(logits) % elt == 0);
  if (!lp_supported(R, V, m, n_top) || stride >= (int64_t)1 << 31) return MOE_ERR_UNSUPPORTED;
  const Span in[] = {span_rows(logits, R, stride * elt, V * elt), {tokens, R * m * 4}};
  const Span outs[] = {{m ? logprobs : nullptr, R * m * 4}, {entropy, R * 4},
                       {top_tokens, R * n_top * 4}, {top_logprobs, R * n_top * 4}};
  MOE_CHECK_ARG(spans_apart(outs, in));
  const LpArgs a = {logits, V, stride, m, tokens, n_top, logprobs, entropy, top_tokens, top_logprobs};
  hipStream_t st = as_stream(stream);
  return dtype == MOE_BF16 ? lp_run<uint16_t>(a, R, st) : lp_run<float>(a, R, st);
}
