// moe_prompt_attention: causal attention of packed sequences.
//
// A block takes one query of one head: 256 keys at a time, a thread a score, then a
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

struct PrArgs {
  const void *q, *k, *v;
  const int32_t *q_offsets, *k_offsets;
  int64_t N, M, B, q_stride, k_stride, v_stride;
  int Hq, Hkv, D;
  float scale2;                                  // scale log2 e
  void* out;
  float* lse;
};

__device__ __forceinline__ float as_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float as_f32(float x) { return x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = f32_to_bf16(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }

__device__ __forceinline__ int64_t pr_offset(const int32_t* o, int64_t b, int64_t n) {
  if (!o) return b == 0 ? 0 : n;
  return min(max((int64_t)o[b], (int64_t)0), n);
}

template <typename Tv>
__global__ void __launch_bounds__(kThreads) pr_simple_kernel(PrArgs a) {
  __shared__ float s_q[256], s_p[kThreads], s_red[kThreads / kWave];
  const int64_t n = blockIdx.x / a.Hq;
  const int h = (int)(blockIdx.x % a.Hq), hk = h / (a.Hq / a.Hkv), t = threadIdx.x;
  int64_t lo = 0, hi = a.B;                      // last sequence that starts at or before n
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if (pr_offset(a.q_offsets, mid, a.N) <= n) lo = mid;
    else hi = mid;
  }
  const int64_t q0 = pr_offset(a.q_offsets, lo, a.N), q1 = pr_offset(a.q_offsets, lo + 1, a.N);
  if (n < q0 || n >= q1) return;
  const int64_t k0 = pr_offset(a.k_offsets, lo, a.M);
  const int64_t k1 = max(k0, pr_offset(a.k_offsets, lo + 1, a.M));
  const int64_t keys = max((int64_t)0, (k1 - k0) - (q1 - q0) + (n - q0) + 1);
  const Tv* const q = static_cast<const Tv*>(a.q) + n * a.q_stride + (int64_t)h * a.D;
  const Tv* const k = static_cast<const Tv*>(a.k) + k0 * a.k_stride + (int64_t)hk * a.D;
  const Tv* const v = static_cast<const Tv*>(a.v) + k0 * a.v_stride + (int64_t)hk * a.D;
  if (t < a.D) s_q[t] = as_f32(q[t]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int64_t j0 = 0; j0 < keys; j0 += kThreads) {
    float s = -INFINITY;
    if (j0 + t < keys) {
      s = 0.f;
      for (int d = 0; d < a.D; ++d) s = fmaf(s_q[d], as_f32(k[(j0 + t) * a.k_stride + d]), s);
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
      for (int64_t j = 0; j < c; ++j) o = fmaf(s_p[j], as_f32(v[(j0 + j) * a.v_stride + t]), o);
    }
    __syncthreads();
  }
  const int64_t at = n * a.Hq + h;
  if (t < a.D) put(static_cast<Tv*>(a.out) + at * a.D + t, l == 0.f ? 0.f : o / l);
  if (a.lse && t == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

bool pr_ok(int64_t N, int64_t M, int64_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype) {
  return N >= 1 && M >= 0 && B >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && D >= 1 &&
         valid_dtype(dtype);
}
bool pr_supported(int64_t N, int64_t M, int64_t B, int32_t Hq, int32_t Hkv, int32_t D) {
  const int64_t lim = (int64_t)1 << 31;
  return D % 8 == 0 && D <= 256 && N < lim / Hq && M < lim && B < lim &&
         (int64_t)Hq * D <= (1 << 24) && N * Hq / 32 + (double)B * Hkv < (1 << 22);
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_prompt_attention_workspace(int64_t N, int64_t M, int64_t B, int32_t Hq,
                                                 int32_t Hkv, int32_t D, int32_t dtype) {
  return 0;
}

extern "C" int moe_prompt_attention(const void* q, const void* k, const void* v, int32_t dtype,
                                    int64_t N, int64_t M, int64_t B, int32_t Hq, int32_t Hkv,
                                    int32_t D, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                    const int32_t* q_offsets, const int32_t* k_offsets, float scale,
                                    void* out, float* lse, void* workspace, size_t ws_bytes,
                                    void* stream) {
  using namespace moe;
  MOE_CHECK_ARG(q && out && pr_ok(N, M, B, Hq, Hkv, D, dtype) && (M == 0 || (k && v)));
  MOE_CHECK_ARG(q_offsets || B == 1);
  MOE_CHECK_ARG(k_offsets || B == 1 || M == N);
  MOE_CHECK_ARG(q_stride >= (int64_t)Hq * D && k_stride >= (int64_t)Hkv * D &&
                v_stride >= (int64_t)Hkv * D);
  MOE_CHECK_ARG(isfinite(scale * kLog2e));       // scores are held times log2 e
  if (!pr_supported(N, M, B, Hq, Hkv, D)) return MOE_ERR_UNSUPPORTED;
  const int64_t elt = dtype == MOE_BF16 ? 2 : 4;
  for (int64_t s : {q_stride, k_stride, v_stride})
    if (s * elt % 16 || s > (1 << 24)) return MOE_ERR_UNSUPPORTED;
  uintptr_t bits = 0;
  for (const void* p : {q, k, v, static_cast<const void*>(out)}) bits |= reinterpret_cast<uintptr_t>(p);
  if (bits & 15) return MOE_ERR_UNSUPPORTED;     // 16-byte loads
  const Span in[] = {span_rows(q, N, q_stride * elt, Hq * D * elt),
                     span_rows(k, M, k_stride * elt, Hkv * D * elt),
                     span_rows(v, M, v_stride * elt, Hkv * D * elt),
                     {q_offsets, (B + 1) * 4}, {k_offsets, (B + 1) * 4}};
  const Span outs[] = {{out, N * Hq * D * elt}, {lse, N * Hq * 4}};
  MOE_CHECK_ARG(spans_apart(outs, in));
  PrArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_offsets = q_offsets;
  a.k_offsets = k_offsets ? k_offsets : B > 1 ? q_offsets : nullptr;
  a.N = N;
  a.M = M;
  a.B = B;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.D = D;
  a.scale2 = scale * kLog2e;
  a.out = out;
  a.lse = lse;
  const dim3 grid((unsigned)(N * Hq));
  hipStream_t st = as_stream(stream);
  if (dtype == MOE_BF16) pr_simple_kernel<uint16_t><<<grid, dim3(kThreads), 0, st>>>(a);
  else pr_simple_kernel<float><<<grid, dim3(kThreads), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}
