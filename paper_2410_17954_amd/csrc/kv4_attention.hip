// moe_kv4_attention: single tokens over a cache in 4 bits.
//
// A block takes one row and query head: 256 keys at a time, a thread a score, then a
// thread a dimension of the values, with the running maximum and sum of the softmax.
#include "moeflow_prompt.h"
#include "common.h"
#include "spans.h"

#include <math.h>

#include <algorithm>

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct KaArgs {
  const void* q;
  const uint8_t *kc, *ks, *vc, *vs;
  const int32_t *cache_row, *lens;
  int64_t R, C, S;
  int Hq, Hkv, D;
  float scale2;
  void* out;
  float* lse;
};

__device__ __forceinline__ float as_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float as_f32(float x) { return x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = f32_to_bf16(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }

__device__ __forceinline__ float value(const uint8_t* codes, const uint8_t* scales, int d) {
  const uint32_t code = codes[d / 2] >> (4 * (d & 1)), c = code & 7u, s = scales[d / 32];
  const float m = c < 4 ? 0.5f * c : c == 7 ? 6.f : (float)c - 2.f;
  return (code & 8u ? -m : m) * (s == 255 ? NAN : __uint_as_float(s << 23));
}

template <typename Tv>
__global__ void __launch_bounds__(kThreads) ka_simple_kernel(KaArgs a) {
  __shared__ float s_q[256], s_p[kThreads], s_red[kThreads / kWave];
  const int64_t r = blockIdx.x / a.Hq;
  const int h = (int)(blockIdx.x % a.Hq), hk = h / (a.Hq / a.Hkv), t = threadIdx.x;
  const int64_t row = a.cache_row ? a.cache_row[r] : r;
  int64_t keys = a.lens ? min(max((int64_t)a.lens[r], (int64_t)0), a.S) : a.S;
  if (row < 0 || row >= a.C) keys = 0;
  const Tv* const q = static_cast<const Tv*>(a.q) + (r * a.Hq + h) * a.D;
  if (t < a.D) s_q[t] = as_f32(q[t]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int64_t j0 = 0; j0 < keys; j0 += kThreads) {
    float s = -INFINITY;
    if (j0 + t < keys) {
      const int64_t at = (row * a.S + j0 + t) * a.Hkv + hk;
      s = 0.f;
      for (int d = 0; d < a.D; ++d)
        s = fmaf(s_q[d], value(a.kc + at * (a.D / 2), a.ks + at * (a.D / 32), d), s);
      s *= a.scale2;
    }
    float top = s;
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, kWave));
    if (lane_id() == 0) s_red[t / kWave] = top;
    __syncthreads();
    for (int w = 0; w < kThreads / kWave; ++w) top = fmaxf(top, s_red[w]);
    top = fmaxf(top, m);
    const float mu = top == -INFINITY ? 0.f : top, f = exp2f(m - mu);
    const float p = j0 + t < keys ? exp2f(s - mu) : 0.f;
    s_p[t] = p;
    float sum = wave_sum(p);
    __syncthreads();
    if (lane_id() == 0) s_red[t / kWave] = sum;
    __syncthreads();
    l *= f;
    o *= f;
    m = top;
    for (int w = 0; w < kThreads / kWave; ++w) l += s_red[w];
    if (t < a.D) {
      const int64_t c = min((int64_t)kThreads, keys - j0);
      for (int64_t j = 0; j < c; ++j) {
        const int64_t at = (row * a.S + j0 + j) * a.Hkv + hk;
        o = fmaf(s_p[j], value(a.vc + at * (a.D / 2), a.vs + at * (a.D / 32), t), o);
      }
    }
    __syncthreads();
  }
  const int64_t at = r * a.Hq + h;
  if (t < a.D) put(static_cast<Tv*>(a.out) + at * a.D + t, l == 0.f ? 0.f : o / l);
  if (a.lse && t == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

bool ka_ok(int64_t R, int64_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  return R >= 1 && S >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && D >= 1;
}
bool ka_supported(int64_t R, int64_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  const int64_t lim = (int64_t)1 << 31;
  return D % 32 == 0 && D <= 256 && R < lim / Hq && S < lim && Hkv < (1 << 24) / D &&
         (double)R * Hkv * (double)ceil_div(Hq / Hkv, 16) < (1 << 22);
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_kv4_attention_workspace(int64_t R, int64_t S, int32_t Hq, int32_t Hkv,
                                              int32_t D) {
  return 0;
}

extern "C" int moe_kv4_attention(const void* q, int32_t dtype, int64_t R, int32_t Hq, int32_t Hkv,
                                 int32_t D, const uint8_t* k_codes, const uint8_t* k_scales,
                                 const uint8_t* v_codes, const uint8_t* v_scales, int64_t C,
                                 int64_t S, const int32_t* cache_row, const int32_t* lens,
                                 float scale, void* out, float* lse, void* workspace,
                                 size_t ws_bytes, void* stream) {
  using namespace moe;
  MOE_CHECK_ARG(q && out && k_codes && k_scales && v_codes && v_scales && valid_dtype(dtype) &&
                C >= 1 && ka_ok(R, S, Hq, Hkv, D));
  MOE_CHECK_ARG(cache_row || R <= C);
  MOE_CHECK_ARG(isfinite(scale * kLog2e));       // scores are held times log2 e
  if (!ka_supported(R, S, Hq, Hkv, D) || C >= (int64_t)1 << 31) return MOE_ERR_UNSUPPORTED;
  if ((double)C * S * Hkv * D > 4e18) return MOE_ERR_UNSUPPORTED;
  uintptr_t bits = 0;
  for (const void* p : {q, static_cast<const void*>(out), static_cast<const void*>(k_codes),
                        static_cast<const void*>(v_codes)})
    bits |= reinterpret_cast<uintptr_t>(p);
  if (bits & 15) return MOE_ERR_UNSUPPORTED;     // 16-byte loads
  const int64_t elt = dtype == MOE_BF16 ? 2 : 4, vals = C * S * Hkv * D;
  const Span in[] = {{q, R * Hq * D * elt}, {k_codes, vals / 2}, {k_scales, vals / 32},
                     {v_codes, vals / 2}, {v_scales, vals / 32}, {cache_row, R * 4}, {lens, R * 4}};
  const Span outs[] = {{out, R * Hq * D * elt}, {lse, R * Hq * 4}};
  MOE_CHECK_ARG(spans_apart(outs, in));
  KaArgs a{};
  a.q = q;
  a.kc = k_codes;
  a.ks = k_scales;
  a.vc = v_codes;
  a.vs = v_scales;
  a.cache_row = cache_row;
  a.lens = lens;
  a.R = R;
  a.C = C;
  a.S = S;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.D = D;
  a.scale2 = scale * kLog2e;
  a.out = out;
  a.lse = lse;
  const dim3 grid((unsigned)(R * Hq));
  hipStream_t st = as_stream(stream);
  if (dtype == MOE_BF16) ka_simple_kernel<uint16_t><<<grid, dim3(kThreads), 0, st>>>(a);
  else ka_simple_kernel<float><<<grid, dim3(kThreads), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}
