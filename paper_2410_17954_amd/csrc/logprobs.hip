// moe_token_logprobs: log-probabilities of given tokens, entropy, best alternatives.
//
// Bound by reading the logits once. A block takes a row, its threads 16 bytes at a time
// in turn, the next ones in flight, and each keeps a reference ref, s = sum e^(z - ref)
// and h = sum e^(z - ref) (z - ref) of what it saw:
//   ln sum e^z = M + ln S,   entropy = ln S - H / S
// with S and H the threads' sums brought to the largest reference M. A reference is
// raised only where a logit exceeds it by more than kSlack, so almost never after the
// first ones.
// Best alternatives need no second pass over the row: of kGroups groups of threads the
// n-th largest of their maxima is a bound T that n logits reach, and only threads whose
// own maximum reaches T hold more of them, about n. A wave reads such a thread's logits
// again, a lane each 16 bytes, and those from T on are ranked by counting.
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
constexpr float kSlack = 8.f;
constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes from an address that is only element-aligned.
struct __attribute__((packed, aligned(2))) Bytes16 { uint32_t w[4]; };

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

// Brings sums to a reference at least as large. No logits: ref -inf, sums 0.
__device__ __forceinline__ void lp_raise(LpSum& x, float to) {
  if (x.ref == to || x.ref == -INFINITY) {
    x.ref = to;
    return;
  }
  const double d = (double)x.ref - (double)to, f = exp(d);
  // a factor that underflows leaves nothing, whatever the difference
  x.h = f > 0.0 || x.s != x.s ? f * (x.h + d * x.s) : 0.0;
  x.s *= f;
  x.ref = to;
}

template <typename Tv, int T>
__global__ void __launch_bounds__(T)
lp_kernel(LpArgs a) {
  using LV = LpVec<Tv>;
  constexpr int VE = LV::N, W = T / kWave, U = 4;
  __shared__ float s_ref[W];
  __shared__ double s_s[W], s_h[W];
  __shared__ __attribute__((aligned(16))) float s_max[kGroups];
  __shared__ float s_thr, s_M;
  __shared__ double s_lnS;
  __shared__ int s_owners, s_count;
  __shared__ int16_t s_owner[T];
  __shared__ float s_key[kKeys];
  __shared__ int32_t s_idx[kKeys];
  const int64_t row = blockIdx.x;
  const Tv* const z = static_cast<const Tv*>(a.logits) + row * a.stride;
  const int t = threadIdx.x, lane = lane_id(), wave = t / kWave;
  const int V = (int)a.V, nvec = V / VE, rest = V - nvec * VE;

  // given tokens: their logits are on the way while the row is
  int32_t tok = -1;
  float ztok = 0.f;
  if (t < a.m) {
    tok = a.tokens[row * a.m + t];
    if (tok >= 0 && tok < V) ztok = LV::one(z + tok);
  }

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
  Bytes16 raw[U];
  auto load = [&](int at) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at + u * T < nvec) raw[u] = *reinterpret_cast<const Bytes16*>(z + (int64_t)(at + u * T) * VE);
  };
  load(t);
  for (int at = t; at < nvec; at += U * T) {
    float v[U][VE];
#pragma unroll
    for (int u = 0; u < U; ++u) LV::unpack(raw[u], v[u]);
    if (at + U * T < nvec) load(at + U * T);
    if (at + (U - 1) * T < nvec) {
      add(&v[0][0], U * VE);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at + u * T < nvec) add(v[u], VE);
    }
  }
  if (t < rest) {
    const float v = LV::one(z + nvec * VE + t);
    add(&v, 1);
  }

  // the block's sums
  float ref = x.ref;
  for (int o = 32; o > 0; o >>= 1) ref = fmaxf(ref, __shfl_xor(ref, o, kWave));
  lp_raise(x, ref);
  x.s = wave_sum(x.s);
  x.h = wave_sum(x.h);
  if (lane == 0) {
    s_ref[wave] = ref;
    s_s[wave] = x.s;
    s_h[wave] = x.h;
  }
  float gmax = best;
  if (T > kGroups) {                             // a group is T / kGroups neighbours
    gmax = fmaxf(gmax, dpp<0xB1>(gmax));
    if (T == 4 * kGroups) gmax = fmaxf(gmax, dpp<0x4E>(gmax));
  }
  if (t % (T / kGroups) == 0) s_max[t / (T / kGroups)] = gmax;
  if (t == 0) s_owners = s_count = 0;
  __syncthreads();
  if (t == 0) {
    float M = s_ref[0];
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, s_ref[w]);
    double S = 0.0, H = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      LpSum y = {s_ref[w], s_s[w], s_h[w]};
      lp_raise(y, M);
      S += y.s;
      H += y.h;
    }
    const bool none = M == -INFINITY && S == 0.0;
    const double lnS = none ? 0.0 : log(S);
    if (a.entropy) a.entropy[row] = none ? 0.f : (float)(lnS - H / S);
    s_M = none ? 0.f : M;
    s_lnS = lnS;                                 // NaN of a row with a NaN or +inf
  }
  if (a.n_top > 0 && t < kGroups) {              // the n-th largest of the groups' maxima
    const float mine = s_max[t];
    int r = 0;
    for (int i = 0; i < kGroups; i += 4) {
      const f32x4_t o = *reinterpret_cast<const f32x4_t*>(s_max + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r += o[e] > mine || (o[e] == mine && i + e < t);
    }
    if (r == a.n_top - 1) s_thr = fmaxf(mine, -FLT_MAX);     // -inf is no candidate
  }
  __syncthreads();
  const float M = s_M;
  const double lnS = s_lnS;
  const bool bad = lnS != lnS;
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
  if (bad) {
    for (int j = t; j < a.n_top; j += T) {
      out_idx[j] = -1;
      out_val[j] = -INFINITY;
    }
    return;
  }
  const float thr = s_thr;
  if (best >= thr) s_owner[atomicAdd(&s_owners, 1)] = (int16_t)t;
  __syncthreads();
  const int owners = s_owners;
  auto offer = [&](float v, int i) {
    if (!(v >= thr)) return;
    const int at = atomicAdd(&s_count, 1);
    if (at < kKeys) {
      s_key[at] = v;
      s_idx[at] = i;
    }
  };
  for (int o = wave; o < owners; o += W) {
    const int own = s_owner[o];
    for (int at = own + lane * T; at < nvec; at += kWave * T) {
      float v[VE];
      LV::unpack(*reinterpret_cast<const Bytes16*>(z + (int64_t)at * VE), v);
#pragma unroll
      for (int i = 0; i < VE; ++i) offer(v[i], at * VE + i);
    }
    if (lane == 0 && own < rest) offer(LV::one(z + nvec * VE + own), nvec * VE + own);
  }
  __syncthreads();
  const int count = s_count;
  if (count <= kKeys) {
    for (int i = t; i < count; i += T) {
      const float v = s_key[i];
      const int32_t id = s_idx[i];
      int r = 0;
      for (int o = 0; o < count; ++o) r += s_key[o] > v || (s_key[o] == v && s_idx[o] < id);
      if (r < a.n_top) {
        out_idx[r] = id;
        out_val[r] = logprob(v);
      }
    }
    for (int j = count + t; j < a.n_top; j += T) {
      out_idx[j] = -1;
      out_val[j] = -INFINITY;
    }
    return;
  }
  // so many equal ones: the best after the one before, again and again over the row
  float pv = INFINITY;
  int pi = -1;
  for (int j = 0; j < a.n_top; ++j) {
    float bv = -INFINITY;
    int bi = 0x7fffffff;
    for (int i = t; i < V; i += T) {
      const float v = LV::one(z + i);
      if (v > -INFINITY && (v < pv || (v == pv && i > pi)) && v > bv) {
        bv = v;
        bi = i;
      }
    }
    for (int o = 32; o > 0; o >>= 1) {
      const float ov = __shfl_xor(bv, o, kWave);
      const int oi = __shfl_xor(bi, o, kWave);
      if (ov > bv || (ov == bv && oi < bi)) {
        bv = ov;
        bi = oi;
      }
    }
    if (lane == 0) {
      s_key[wave] = bv;
      s_idx[wave] = bi;
    }
    __syncthreads();
    bv = s_key[0];
    bi = s_idx[0];
#pragma unroll
    for (int w = 1; w < W; ++w)
      if (s_key[w] > bv || (s_key[w] == bv && s_idx[w] < bi)) {
        bv = s_key[w];
        bi = s_idx[w];
      }
    if (t == 0) {
      const bool got = bi != 0x7fffffff;
      out_idx[j] = got ? bi : -1;
      out_val[j] = got ? logprob(bv) : -INFINITY;
    }
    pv = bv;
    pi = bi;
    __syncthreads();                             // s_key is rewritten next
  }
}

bool lp_ok(int64_t R, int64_t V, int64_t m, int32_t n_top) {
  return R >= 1 && V >= 1 && m >= 0 && n_top >= 0;
}
bool lp_supported(int64_t R, int64_t V, int64_t m, int32_t n_top) {
  return n_top <= kMaxTop && V <= (1 << 24) && R < (1 << 22) && m < ((int64_t)1 << 31) / R;
}

template <typename Tv>
int lp_run(const LpArgs& a, int64_t R, hipStream_t st) {
  if (R <= 256) lp_kernel<Tv, 1024><<<dim3((unsigned)R), dim3(1024), 0, st>>>(a);
  else lp_kernel<Tv, 256><<<dim3((unsigned)R), dim3(256), 0, st>>>(a);
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
