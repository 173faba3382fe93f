// moe_token_logprobs: log-probabilities of given tokens, entropy, best alternatives.
//
// A block takes a row: its maximum, its sums, then one pass a top token.
#include "moeflow_prompt.h"
#include "common.h"
#include "spans.h"

#include <math.h>

#include <algorithm>

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTop = 64;

__device__ __forceinline__ float as_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float as_f32(float x) { return x; }

template <typename Tv>
__global__ void __launch_bounds__(kThreads)
lp_simple_kernel(const Tv* logits, int64_t V, int64_t stride, const int32_t* tokens, int64_t m,
                 int n_top, float* logprobs, float* entropy, int32_t* top_tokens,
                 float* top_logprobs) {
  __shared__ float s_v[kThreads];
  __shared__ int32_t s_i[kThreads];
  __shared__ double s_s[kThreads], s_h[kThreads];
  const int64_t r = blockIdx.x;
  const Tv* const z = logits + r * stride;
  const int t = threadIdx.x;
  float top = -INFINITY;
  bool bad = false;
  for (int64_t i = t; i < V; i += kThreads) {
    const float x = as_f32(z[i]);
    bad |= !(x < INFINITY);
    top = fmaxf(top, x);
  }
  s_v[t] = top;
  s_i[t] = bad;
  __syncthreads();
  for (int i = 0; i < kThreads; ++i) {
    top = fmaxf(top, s_v[i]);
    bad |= s_i[i] != 0;
  }
  __syncthreads();
  const bool none = !bad && top == -INFINITY;
  double s = 0.0, h = 0.0;
  for (int64_t i = t; i < V; i += kThreads) {
    const float x = as_f32(z[i]);
    if (x == -INFINITY || bad) continue;
    const double d = (double)x - top;
    const double e = (double)__expf((float)d);
    s += e;
    if (e > 0) h += e * d;
  }
  s_s[t] = s;
  s_h[t] = h;
  __syncthreads();
  s = h = 0.0;
  for (int i = 0; i < kThreads; ++i) {
    s += s_s[i];
    h += s_h[i];
  }
  // the difference to the maximum first: beside a mask's lowest number ln S is lost
  const double off = none ? 0.0 : (double)top, ls = bad ? (double)NAN : none ? 0.0 : log(s);
  for (int64_t j = t; j < m; j += kThreads) {
    const int64_t v = tokens[r * m + j];
    const bool in = v >= 0 && v < V;
    logprobs[r * m + j] = !in ? -INFINITY : (float)((double)as_f32(z[v]) - off - ls);
  }
  if (entropy && t == 0) entropy[r] = bad ? NAN : none ? 0.f : (float)(ls - h / s);
  float pv = INFINITY;
  int32_t pi = -1;
  for (int j = 0; j < n_top; ++j) {
    float bv = -INFINITY;
    int32_t bi = 0x7fffffff;
    if (!bad)
      for (int64_t i = t; i < V; i += kThreads) {
        const float x = as_f32(z[i]);
        if (x == -INFINITY || !(x < pv || (x == pv && i > pi))) continue;
        if (x > bv) {
          bv = x;
          bi = (int32_t)i;
        }
      }
    __syncthreads();
    s_v[t] = bv;
    s_i[t] = bi;
    __syncthreads();
    for (int i = 0; i < kThreads; ++i)
      if (s_v[i] > bv || (s_v[i] == bv && s_i[i] < bi)) {
        bv = s_v[i];
        bi = s_i[i];
      }
    if (t == 0) {
      const bool got = bi != 0x7fffffff;
      top_tokens[r * n_top + j] = got ? bi : -1;
      top_logprobs[r * n_top + j] = got ? (float)((double)bv - off - ls) : -INFINITY;
    }
    pv = bv;
    pi = bi;
  }
}

bool lp_ok(int64_t R, int64_t V, int64_t m, int32_t n_top) {
  return R >= 1 && V >= 1 && m >= 0 && n_top >= 0;
}
bool lp_supported(int64_t R, int64_t V, int64_t m, int32_t n_top) {
  return n_top <= kMaxTop && V <= (1 << 24) && R < (1 << 22) && m < ((int64_t)1 << 31) / R;
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
  hipStream_t st = as_stream(stream);
  const dim3 grid((unsigned)R), block(kThreads);
  if (dtype == MOE_BF16)
    lp_simple_kernel<<<grid, block, 0, st>>>(static_cast<const uint16_t*>(logits), V, stride,
                                             tokens, m, n_top, logprobs, entropy, top_tokens,
                                             top_logprobs);
  else
    lp_simple_kernel<<<grid, block, 0, st>>>(static_cast<const float*>(logits), V, stride, tokens,
                                             m, n_top, logprobs, entropy, top_tokens,
                                             top_logprobs);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}
