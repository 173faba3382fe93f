// A cache of keys and values in 4 bits: moe_kv4_store, moe_kv4_load.
//
// Both are copies bound by HBM. A thread takes 8 channels of a key and of its value (16
// bytes of bf16 <-> one word of codes), four neighbouring threads a block of 32; they
// find its largest magnitude with two moves within a quad, and the first of them writes
// the scale.
#include "moeflow_prompt.h"
#include "common.h"
#include "rows.h"
#include "spans.h"

#include <algorithm>

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int kMinExp = -124, kMaxExp = 125;
constexpr uint8_t kNaNScale = 255;

struct Kv4Args {
  const void *k, *v;                             // of a load: written
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  const int32_t* slots;
  int64_t N, n_slots, k_stride, v_stride, pieces; // pieces: of 8 channels, of k, and of v
  int row;                                       // pieces of a token
};

// Bits of a nonnegative float -> the biased exponent of its block: least e with
// x <= 1.75 * 4 * 2^e, that is e = exponent(x) - 2, one more above 1.75 * 2^exponent.
__device__ __forceinline__ int kv4_scale(uint32_t amax) {
  if (amax >= 0x7f800000u) return kNaNScale;
  const int e = (int)(amax >> 23) - 127 - 2 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kMinExp), kMaxExp) + 127;
}

typedef __attribute__((ext_vector_type(2))) float f32x2_t;

// Codes of eight channels over 2^e: the conversion rounds to the nearest, ties to the even
// code, and takes what is larger as 6.
__device__ __forceinline__ uint32_t kv4_codes(const float (&x)[8], float unit) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
}

// The values of eight codes; those of a scale of 255 are NaN.
__device__ __forceinline__ void kv4_values(uint32_t w, uint32_t scale, float (&x)[8]) {
  const float unit = __uint_as_float(scale << 23);
  const f32x2_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3)};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = v[i][0];
    x[2 * i + 1] = v[i][1];
  }
}

template <typename Tv> struct Eight;
template <> struct Eight<uint16_t> {
  static __device__ __forceinline__ void get(const uint16_t* p, float (&x)[8]) {
    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void put(uint16_t* p, const float (&x)[8]) {
    u32x4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (uint32_t)f32_to_bf16(x[2 * i]) | (uint32_t)f32_to_bf16(x[2 * i + 1]) << 16;
    *reinterpret_cast<u32x4_t*>(p) = w;
  }
};
template <> struct Eight<float> {
  static __device__ __forceinline__ void get(const float* p, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x4_t w = reinterpret_cast<const f32x4_t*>(p)[j];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * j + i] = w[i];
    }
  }
  static __device__ __forceinline__ void put(float* p, const float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      reinterpret_cast<f32x4_t*>(p)[j] = f32x4_t{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
  }
};

// Piece, token and slot of a thread; false: nothing to do. A block's four threads share a
// token.
__device__ __forceinline__ bool kv4_find(const Kv4Args& a, int64_t& n, uint32_t& c, int64_t& slot) {
  const uint32_t at = blockIdx.x * (uint32_t)kThreads + threadIdx.x;
  if (at >= (uint32_t)a.pieces) return false;
  n = at / (uint32_t)a.row;
  c = at - (uint32_t)n * (uint32_t)a.row;
  slot = a.slots ? a.slots[n] : n;
  return slot >= 0 && slot < a.n_slots;
}

template <typename Tv>
__global__ void __launch_bounds__(kThreads) kv4_store_kernel(Kv4Args a) {
  int64_t n, slot;
  uint32_t c;
  if (!kv4_find(a, n, c, slot)) return;
  float x[2][8];
  Eight<Tv>::get(static_cast<const Tv*>(a.k) + n * a.k_stride + c * 8, x[0]);
  Eight<Tv>::get(static_cast<const Tv*>(a.v) + n * a.v_stride + c * 8, x[1]);
  const int64_t to = slot * a.row + c;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[i][j]) & 0x7fffffffu);
    top = max(top, (uint32_t)dpp<0xB1>((int)top));
    top = max(top, (uint32_t)dpp<0x4E>((int)top));
    const int s = kv4_scale(top);
    reinterpret_cast<uint32_t*>(i ? a.v_codes : a.k_codes)[to] =
        s == kNaNScale ? 0 : kv4_codes(x[i], __uint_as_float((uint32_t)s << 23));
    if ((c & 3) == 0) (i ? a.v_scales : a.k_scales)[to >> 2] = (uint8_t)s;
  }
}

template <typename Tv>
__global__ void __launch_bounds__(kThreads) kv4_load_kernel(Kv4Args a) {
  int64_t n, slot;
  uint32_t c;
  if (!kv4_find(a, n, c, slot)) return;
  const int64_t from = slot * a.row + c;
  const uint32_t wk = reinterpret_cast<const uint32_t*>(a.k_codes)[from];
  const uint32_t wv = reinterpret_cast<const uint32_t*>(a.v_codes)[from];
  const uint32_t sk = a.k_scales[from >> 2], sv = a.v_scales[from >> 2];
  float x[8];
  kv4_values(wk, sk, x);
  Eight<Tv>::put(const_cast<Tv*>(static_cast<const Tv*>(a.k)) + n * a.k_stride + c * 8, x);
  kv4_values(wv, sv, x);
  Eight<Tv>::put(const_cast<Tv*>(static_cast<const Tv*>(a.v)) + n * a.v_stride + c * 8, x);
}

int kv4_run(bool load, int32_t dtype, const Kv4Args& a, int32_t Hkv, int32_t D, void* stream) {
  MOE_CHECK_ARG(a.k && a.v && a.k_codes && a.k_scales && a.v_codes && a.v_scales &&
                valid_dtype(dtype) && a.N >= 1 && a.n_slots >= 1 && Hkv >= 1 && D >= 1);
  MOE_CHECK_ARG(a.slots || a.N <= a.n_slots);
  const int64_t lim = (int64_t)1 << 31, elt = dtype == MOE_BF16 ? 2 : 4;
  if (D % 32 || D > 256 || Hkv > (1 << 24) / D || a.N >= lim / Hkv || a.n_slots >= lim)
    return MOE_ERR_UNSUPPORTED;
  const int64_t row = (int64_t)Hkv * D;
  MOE_CHECK_ARG(a.k_stride >= row && a.v_stride >= row);
  if (a.N * row >= (int64_t)1 << 34) return MOE_ERR_UNSUPPORTED;
  for (int64_t s : {a.k_stride, a.v_stride})
    if (s * elt % 16 || s > (1 << 24)) return MOE_ERR_UNSUPPORTED;
  uintptr_t bits = 0;
  for (const void* p : {a.k, a.v, static_cast<const void*>(a.k_codes),
                        static_cast<const void*>(a.v_codes)})
    bits |= reinterpret_cast<uintptr_t>(p);
  if (bits & 15) return MOE_ERR_UNSUPPORTED;     // 16-byte loads
  const Span k = span_rows(a.k, a.N, a.k_stride * elt, row * elt);
  const Span v = span_rows(a.v, a.N, a.v_stride * elt, row * elt);
  const Span idx = {a.slots, a.N * 4};
  const Span cache[] = {{a.k_codes, a.n_slots * row / 2}, {a.k_scales, a.n_slots * row / 32},
                        {a.v_codes, a.n_slots * row / 2}, {a.v_scales, a.n_slots * row / 32}};
  if (load) {
    const Span in[] = {cache[0], cache[1], cache[2], cache[3], idx}, to_k[] = {k}, to_v[] = {v};
    MOE_CHECK_ARG(spans_apart(to_k, in) && spans_apart(to_v, in));
    MOE_CHECK_ARG(!rows_meet(a.k, a.v, a.N, a.k_stride * elt, a.v_stride * elt, row * elt));
  } else {
    const Span in[] = {k, v, idx};
    MOE_CHECK_ARG(spans_apart(cache, in));
  }
  Kv4Args b = a;
  b.row = (int)(row / 8);
  b.pieces = a.N * b.row;
  const dim3 grid((unsigned)ceil_div(b.pieces, kThreads));
  hipStream_t st = as_stream(stream);
  if (load) {
    if (dtype == MOE_BF16) kv4_load_kernel<uint16_t><<<grid, dim3(kThreads), 0, st>>>(b);
    else kv4_load_kernel<float><<<grid, dim3(kThreads), 0, st>>>(b);
  } else {
    if (dtype == MOE_BF16) kv4_store_kernel<uint16_t><<<grid, dim3(kThreads), 0, st>>>(b);
    else kv4_store_kernel<float><<<grid, dim3(kThreads), 0, st>>>(b);
  }
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

}  // namespace
}  // namespace moe

extern "C" int moe_kv4_store(const void* k, const void* v, int32_t dtype, int64_t N, int32_t Hkv,
                             int32_t D, int64_t k_stride, int64_t v_stride, const int32_t* slots,
                             int64_t n_slots, uint8_t* k_codes, uint8_t* k_scales,
                             uint8_t* v_codes, uint8_t* v_scales, void* stream) {
  const moe::Kv4Args a = {k, v, k_codes, k_scales, v_codes, v_scales, slots, N, n_slots,
                          k_stride, v_stride, 0, 0};
  return moe::kv4_run(false, dtype, a, Hkv, D, stream);
}

extern "C" int moe_kv4_load(const uint8_t* k_codes, const uint8_t* k_scales,
                            const uint8_t* v_codes, const uint8_t* v_scales, int64_t n_slots,
                            const int32_t* slots, int64_t N, int32_t Hkv, int32_t D, int32_t dtype,
                            int64_t k_stride, int64_t v_stride, void* k, void* v, void* stream) {
  const moe::Kv4Args a = {k, v, const_cast<uint8_t*>(k_codes), const_cast<uint8_t*>(k_scales),
                          const_cast<uint8_t*>(v_codes), const_cast<uint8_t*>(v_scales), slots, N,
                          n_slots, k_stride, v_stride, 0, 0};
  return moe::kv4_run(true, dtype, a, Hkv, D, stream);
}
