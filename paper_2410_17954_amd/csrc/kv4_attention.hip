// moe_kv4_attention: single tokens over a cache in 4 bits.
//
// Bound by reading the cache once (HBM): 17/32 byte a value.
//   S^T = K Q^T     rows: keys, columns: the query heads of a key head
//   O^T = V^T P^T   rows: values' dimensions, columns: query heads
// A wave takes 64 keys of one head at a time. Their codes go straight from memory to
// LDS, four lanes a key (lanes that load from sixteen keys each keep the address unit
// busy four times as long), the next keys while the values are in work and the other
// way round. A compute unit holds sixteen waves by registers and LDS (bf16, D of 128);
// splits stop at two blocks of it, eight waves, which keep up to 68 KB on their way. Keys
// come back as MFMA operands, a quarter of a head a lane (k slots 8t + j of quarter q4 are
// dimensions q4 D/4 + 8t + j, of the queries too), and become bf16 with their block's
// scale, two an instruction: exact, as a value has two bits times a power of two. Rows of
// the score tiles are dealt so that lane (query r, q4) holds scores of keys 16 q4 .. 16 q4 + 15,
// which is what a transposing read of 4-bit values gives a lane: 16 keys of one
// dimension. Values stay unscaled there; a key's scales go into the numerators, once
// for every 32 dimensions, exact as well.
// float32 queries and numerators are cut into three bf16 numbers of 8 bits each,
// whose products are exact: three MFMAs for one, which the cache's stream hides.
// The waves of a block are neighbouring heads over the same keys, which share cache
// lines, and where there are fewer heads ranges of keys, added up through LDS at the
// end. Long key ranges are split over blocks, and a second launch joins the splits.
#include "moeflow_prompt.h"
#include "attention.h"
#include "dma.h"
#include "spans.h"

#include <algorithm>

namespace moe {
namespace {

constexpr int KEYS = 64, KT = 4;                 // of a wave's step
constexpr uint32_t kPastEnd = 0x7ffffff0u;       // no buffer here is as long

struct KaArgs {
  const void* q;
  const uint8_t *codes[2], *scales[2];           // of keys, of values
  const int32_t *cache_row, *lens;
  int64_t R, C, S;
  int Hq, Hkv, D, nq, tiles, heads;              // tiles: of 16 query heads of a key head;
                                                 // heads: key heads of a block
  float scale2;
  uint32_t keep, flip;
  int splits;
  float* part_o;                                 // [splits][R * Hq][D]
  float2* part_ml;                               // [splits][R * Hq]
  void* out;
  float* lse;
};

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// Eight codes of a word times a scale, as an MFMA operand.
__device__ __forceinline__ u32x4_t eight_bf16(uint32_t w, float scale) {
  u32x4_t x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return x;
}

// x as a sum of NS bf16 numbers: cut, not rounded, so that three hold all 24 bits. Of an
// infinity the first part is one and the others are NaN.
template <int NS>
__device__ __forceinline__ void cut(float x, uint16_t (&part)[NS]) {
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const uint32_t top = __float_as_uint(x) & 0xffff0000u;
    part[n] = (uint16_t)(top >> 16);
    x -= __uint_as_float(top);
  }
}

__device__ __forceinline__ void mfma(f32x4_t& c, const u32x4_t& x, const u32x4_t& y) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x),
                                              __builtin_bit_cast(bf16x8_t, y), c, 0, 0, 0);
}

typedef __attribute__((ext_vector_type(2))) int i32x2_t;
typedef __attribute__((address_space(3))) i32x2_t lds_i32x2_t;
typedef __attribute__((ext_vector_type(8))) uint16_t u16x8_t;

// DP: the dimension padded to 64, 128 or 256; channels past D are zeros. EACH: scales of a
// key that a load takes, what D / 32 is a multiple of (a word of the buffer is read as
// a whole or not at all).
template <typename Tv, int DP, int EACH>
struct KaCore {
  static constexpr bool BF16 = sizeof(Tv) == 2;
  static constexpr int NS = BF16 ? 1 : 3;        // bf16 numbers of a query's channel
  static constexpr int WN = DP / 32;             // words of a lane's quarter, k-steps of S
  static constexpr int NB = DP / 32;             // blocks of a key
  static constexpr int PC = DP / 32;             // 16-byte pieces of a key's codes
  static constexpr int kCodes = KEYS * DP / 2, NI = kCodes / 1024;   // of a step; its loads
  // fewest loads of a step's scales, and their words: of D / 32 in (DP / 64, DP / 32]
  static constexpr int NSI = DP == 64 ? 1 : EACH == 1 ? DP / 64 + 1 : EACH == 2 ? 3 : DP / 128;
  static constexpr int kRaw = (DP == 64 ? 1 : EACH == 1 ? NB - 1 : NSI) * KEYS * 4;
  static constexpr int NBV = kRaw / (KEYS * 4) * EACH, DT = 2 * NBV;   // blocks of D at most, tiles of O
  static constexpr int kGroup = NI + NSI;        // loads of a step's keys, or of its values
  static constexpr int kSlot = kCodes + kRaw;    // keys, or values
  static constexpr int kUnits = KEYS * NBV * 4;  // float scales of a step's values
  static constexpr int kLds = 2 * kSlot + kUnits;

  // Piece p of key k lies at p ^ swz, so that the reads of sixteen lanes meet different
  // banks: of keys 16 (r >> 2) + 4 kt + (r & 3), of values 16 q4 + r.
  static __device__ __forceinline__ int swz_k(int k) {
    return PC == 2 ? (k >> 4) & 1 : PC == 4 ? (k >> 4) & 3 : (k >> 1 & 1) | (k >> 3 & 6);
  }
  static __device__ __forceinline__ int swz_v(int k) {
    return PC == 2 ? (k >> 3) & 1 : PC == 4 ? (k >> 2) & 3 : (k >> 1) & 7;
  }
  // Byte offsets of what a lane loads, from a step's first key on.
  static __device__ __forceinline__ void offsets(uint32_t (&off)[2][NI], const KaArgs& a) {
    const uint32_t row = (uint32_t)(a.Hkv * (a.D / 2));
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int g = i * 64 + lane_id(), k = g / PC, p = g % PC;
      const int pk = p ^ swz_k(k), pv = p ^ swz_v(k);
      off[0][i] = pk * 32 < a.D ? k * row + pk * 16 : kPastEnd;
      off[1][i] = pv * 32 < a.D ? k * row + pv * 16 : kPastEnd;
    }
  }
  // n keys from `key` on: codes, then a word a key of EACH scales at a time.
  static __device__ __forceinline__ void load(uint32_t lds, const uint8_t* codes, const uint8_t* scales,
                                              int64_t key, int n, const uint32_t (&off)[NI],
                                              const KaArgs& a) {
    const int nb = a.D / 32;
    const u32x4_t rc = dma_rows(codes, key, n, (uint32_t)(a.Hkv * nb * 16), (uint32_t)nb * 16);
    const u32x4_t rs = dma_rows(scales, key, n, (uint32_t)(a.Hkv * nb), (uint32_t)nb);
#pragma unroll
    for (int i = 0; i < NI; ++i) dma<16>(lds + i * 1024, off[i], rc);
    const uint32_t at = (uint32_t)lane_id() * (uint32_t)(a.Hkv * nb);
#pragma unroll
    for (int i = 0; i < kRaw / (KEYS * 4); ++i)
      if (i < NSI || i * EACH < nb) dma<EACH>(lds + kCodes + i * KEYS * 4, at + i * EACH, rs);
  }
  // Values' scales as floats, [block][key]; 255 is NaN.
  static __device__ __forceinline__ void units(char* to, const char* raw) {
    const uint32_t* const from = reinterpret_cast<const uint32_t*>(raw) + lane_id();
    float* const out = reinterpret_cast<float*>(to) + lane_id();
#pragma unroll
    for (int i = 0; i < kRaw / (KEYS * 4); ++i) {
      const uint32_t w = from[i * KEYS];
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const uint32_t s = (w >> (8 * e)) & 255u;
        out[(i * EACH + e) * KEYS] = s == 255u ? NAN : __uint_as_float(s << 23);
      }
    }
  }
  static __device__ __forceinline__ void scores(f32x4_t (&s)[1][KT], const u32x4_t (&q)[NS][WN],
                                                const char* codes, int D) {
    const int r = lane_id() & 15, q4 = lane_id() >> 4;
    // a scale of 255 makes the conversion NaN; codes past D are zeros, under the scale
    // of a block that there is
    auto unit = [&](int k, int b) {
      b = min(b, D / 32 - 1);
      const uint8_t s = static_cast<uint8_t>(codes[kCodes + (b / EACH * KEYS + k) * 4 + b % EACH]);
      return __uint_as_float((uint32_t)s << 23);
    };
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) s[0][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      uint32_t w[WN];
      float u[DP == 256 ? 2 : 1];
      const int k = 16 * (r >> 2) + 4 * kt + (r & 3);
      const char* const row = codes + k * (DP / 2);
      if constexpr (DP == 64) {
        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(row + ((q4 >> 1) ^ swz_k(k)) * 16 + (q4 & 1) * 8);
        w[0] = x[0];
        w[1] = x[1];
        u[0] = unit(k, q4 >> 1);
      } else {
#pragma unroll
        for (int i = 0; i < WN / 4; ++i) {
          const int p = WN / 4 * q4 + i;
          const u32x4_t x = *reinterpret_cast<const u32x4_t*>(row + (p ^ swz_k(k)) * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[4 * i + e] = x[e];
          u[i] = unit(k, p);
        }
      }
#pragma unroll
      for (int t = 0; t < WN; ++t) {
        const u32x4_t x = eight_bf16(w[t], u[DP == 256 ? t / 4 : 0]);
#pragma unroll
        for (int n = 0; n < NS; ++n) mfma(s[0][kt], x, q[n][t]);
      }
    }
  }
  // O += V^T P^T. bf16: p is rounded to bf16 (by at most 2^-8 of it, for the matrix cores);
  // its sum is taken of the float32 values. Of flat attention over 1000 or 8192 keys the
  // result is off by 2.3e-3 (rms), 1.7e-3 of it the rounding of the result itself; with p
  // as the sum of two bf16 numbers only that is left, and one row of 131072 keys takes
  // 39.6 us for 34.7, 64 of 8192 119 for 116, 200 of 777 44.6 for 39.5.
  static __device__ __forceinline__ void values(f32x4_t (&o)[1][DT], const f32x4_t (&p)[1][KT],
                                                const char* codes, const char* units) {
    const int r = lane_id() & 15, q4 = lane_id() >> 4, k = 16 * q4 + r;
#pragma unroll
    for (int b = 0; b < NBV; ++b) {
      i32x2_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)                // 32 dimensions are one piece
        w[i] = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
            (lds_i32x2_t*)(codes + k * (DP / 2) + (b ^ swz_v(k)) * 16 + 8 * i));
      u32x4_t pb[2][NS];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        f32x4_t ps[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
          ps[i] = p[0][2 * j + i] * *reinterpret_cast<const f32x4_t*>(
                                        units + (b * KEYS + 16 * q4 + 8 * j + 4 * i) * 4);
        if constexpr (BF16) {
          bf16x8_t x;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = (__bf16)ps[e / 4][e % 4];
          pb[j][0] = __builtin_bit_cast(u32x4_t, x);
        } else {
          u16x8_t x[NS];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            uint16_t part[NS];
            cut<NS>(ps[e / 4][e % 4], part);
#pragma unroll
            for (int n = 0; n < NS; ++n) x[n][e] = part[n];
          }
#pragma unroll
          for (int n = 0; n < NS; ++n) pb[j][n] = __builtin_bit_cast(u32x4_t, x[n]);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x4_t v = eight_bf16((uint32_t)w[i][j], 1.f);
#pragma unroll
          for (int n = 0; n < NS; ++n) mfma(o[0][2 * b + i], v, pb[j][n]);
        }
    }
  }
};

// Waves of a block, of which a compute unit holds four.
constexpr int ka_waves(int dp) { return dp == 256 ? 2 : 4; }

// Waves a SIMD, the most that leave no spilled register.
constexpr int ka_occupancy(int elt, int dp, int each) {
  return dp == 256 ? (elt == 4 ? 1 : 2) : elt == 4 ? 2 : dp == 128 && each == 1 ? 3 : 4;
}

template <typename Tv, int DP, int EACH>
__global__ void __launch_bounds__(64 * ka_waves(DP), ka_occupancy(sizeof(Tv), DP, EACH))
ka_kernel(KaArgs a) {
  using C = KaCore<Tv, DP, EACH>;
  constexpr int DT = C::DT, W = ka_waves(DP);
  __shared__ __attribute__((aligned(16))) char lds[W * C::kLds];
  __shared__ float s_m[W][16], s_l[W][16];
  static_assert(C::kLds >= DT * kWave * 16, "O of a wave");
  const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // Block b runs on XCD b % 8: the groups of heads of a unit (row, split, tile), which lie
  // next to each other in a cache, go to one XCD.
  const int hw = a.heads, kw = W / hw;
  const uint32_t groups = (uint32_t)(a.Hkv / hw);
  const uint32_t v = blockIdx.x / (8 * groups) * 8 + blockIdx.x % 8;
  const int h = (int)(blockIdx.x / 8 % groups) * hw + wave % hw, tile = (int)(v % a.tiles);
  const int split = (int)(v / a.tiles % a.splits), sub = wave / hw;
  const int64_t row = v / (a.tiles * a.splits);
  if (row >= a.R) return;
  const int64_t from = a.cache_row ? (int64_t)a.cache_row[row] : row;
  uint32_t len = (uint32_t)(a.lens ? min(max((int64_t)a.lens[row], (int64_t)0), a.S) : a.S);
  if (from < 0 || from >= a.C) len = 0;
  const uint32_t per = ((len + a.splits - 1) / a.splits + KEYS - 1) / KEYS * KEYS;
  const int lo = (int)min((uint64_t)len, (uint64_t)per * split), hi = (int)min(len, lo + per);
  const int cols = min(a.nq - tile * 16, 16);
  const int64_t RH = a.R * a.Hq, at = row * a.Hq + h * a.nq + tile * 16 + r, to = split * RH + at;
  if (lo >= hi && a.splits > 1) {                // no keys: this split adds nothing
    if (sub == 0 && q4 == 0 && r < cols) a.part_ml[to] = make_float2(-INFINITY, 0.f);
    return;
  }
  const int64_t base = (from * a.S * a.Hkv + h) * (a.D / 32);   // of the scales; codes 16 a block
  char* const mine = lds + wave * C::kLds;
  const uint32_t mine_at = lds_address(mine);
  char* const units = mine + 2 * C::kSlot;
  uint32_t off[2][C::NI];
  C::offsets(off, a);
  const int steps = (int)(((uint32_t)(hi - lo) + KEYS - 1) / KEYS);
  auto load = [&](int x, int st) {               // keys (x = 0) or values (1) of a step
    const int key = lo + st * KEYS;
    C::load(mine_at + x * C::kSlot, a.codes[x] + base * 16, a.scales[x] + base, key,
            min(hi - key, KEYS), off[x], a);
  };
  u32x4_t q[C::NS][C::WN];
  float q_top = 0.f;
#pragma unroll
  for (int t = 0; t < C::WN; ++t) {
    const int d = q4 * (DP / 4) + 8 * t;
    const bool in = r < cols && d < a.D;
    const Tv* const src = static_cast<const Tv*>(a.q) + (in ? at * a.D + d : 0);
    if constexpr (C::BF16) {
      q[0][t] = u32x4_t{0, 0, 0, 0};
      if (in) q[0][t] = (*reinterpret_cast<const u32x4_t*>(src) & a.keep) ^ a.flip;
    } else {
      u32x4_t x[2] = {};
      if (in)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          x[i] = (reinterpret_cast<const u32x4_t*>(src)[i] & a.keep) ^ a.flip;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x0 = __uint_as_float(x[j / 2][2 * (j % 2)]);
        const float x1 = __uint_as_float(x[j / 2][2 * (j % 2) + 1]);
        uint16_t p0[C::NS], p1[C::NS];
        cut<C::NS>(x0, p0);
        cut<C::NS>(x1, p1);
        q_top = fmaxf(q_top, fmaxf(fabsf(x0), fabsf(x1)));
#pragma unroll
        for (int n = 0; n < C::NS; ++n) q[n][t][j] = (uint32_t)p0[n] | (uint32_t)p1[n] << 16;
      }
    }
  }
  // All of an infinite channel is in its first part. Looked for once a lane: a selection
  // for every channel took 0.3 us of a call.
  if (!C::BF16 && q_top == INFINITY) {
#pragma unroll
    for (int t = 0; t < C::WN; ++t) {
      const int d = q4 * (DP / 4) + 8 * t;
      if (d >= a.D) continue;
      const float* const src = static_cast<const float*>(a.q) + at * a.D + d;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (fabsf(src[j]) == INFINITY)
#pragma unroll
          for (int n = 1; n < C::NS; ++n) q[n][t][j / 2] &= j % 2 ? 0xffffu : 0xffff0000u;
    }
  }
  f32x4_t o[1][DT];
  float m_run[1] = {-INFINITY}, l_run[1] = {0.f};
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[0][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // the next step's keys are loaded as soon as the scores have used this step's, its
  // values after the second product
  constexpr int G = C::kGroup;
  if (sub < steps) {
    load(0, sub);
    load(1, sub);
  }
  const char* const kc = mine;
  const char* const vc = mine + C::kSlot;
  for (int st = sub; st < steps; st += kw) {
    const bool one = st + kw < steps;            // one more step
    wait_loads<G>();
    f32x4_t s[1][KT];
    C::scores(s, q, kc, a.D);
    wait_lds();
    if (one) load(0, st + kw);
    const int keys = min(hi - lo - st * KEYS, KEYS);
    if (keys < KEYS) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * q4 + 4 * kt + e >= keys) s[0][kt][e] = -INFINITY;
    }
    softmax_step<Tv>(s, m_run, l_run, o, a.scale2);
    if (one) wait_loads<G>();
    else wait_loads<0>();
    C::units(units, vc + C::kCodes);
    C::values(o, s, vc, units);
    wait_lds();
    if (one) load(1, st + kw);
  }
  // join the waves of a head: common maximum, then O through LDS
  float top = m_run[0], l = quad_sum(l_run[0]);
  if (kw > 1) {
    if (q4 == 0) {
      s_m[wave][r] = top;
      s_l[wave][r] = l;
    }
    __syncthreads();                             // and every wave is done with its codes
    f32x4_t* const part = reinterpret_cast<f32x4_t*>(lds);
    const int w0 = wave % hw;
    for (int i = 0; i < kw; ++i) top = fmaxf(top, s_m[w0 + i * hw][r]);
    const float mu = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m_run[0] - mu);
    l = 0.f;
    for (int i = 0; i < kw; ++i) l += s_l[w0 + i * hw][r] * __builtin_amdgcn_exp2f(s_m[w0 + i * hw][r] - mu);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) part[(wave * DT + dt) * kWave + lane] = o[0][dt] * f;
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      o[0][dt] = part[(w0 * DT + dt) * kWave + lane];
      for (int i = 1; i < kw; ++i) o[0][dt] += part[((w0 + i * hw) * DT + dt) * kWave + lane];
    }
  }
  if (r >= cols) return;
  if (q4 == 0) {
    // keys without weight may have values of NaN: their sum, of a maximum of -inf, adds 0
    if (a.splits > 1) a.part_ml[to] = make_float2(top, l == 0.f ? 1.f : l);
    else if (a.lse) a.lse[at] = lse_of(top, l);
  }
  const float inv = 1.f / l;                     // of no weight: 0, whatever the values hold
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const int d = 16 * dt + 4 * q4;              // D is a multiple of 32
    if (d >= a.D) continue;
    if (a.splits > 1) *reinterpret_cast<f32x4_t*>(a.part_o + to * a.D + d) = o[0][dt];
    else put4(static_cast<Tv*>(a.out) + at * a.D + d,
              l == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : o[0][dt] * inv);
  }
}

struct KaPlan {
  int heads, tiles, splits;
  int64_t blocks;
  size_t ml, total;
};

// Blocks wanted, two a compute unit: twice as many cost 3 to 12 % of long calls, whose
// joins grow. Fewer than kMinKeys keys a split do not earn the join (one row of 777 keys
// 9.4 us with splits of 128, 10.4 of 256, 12.4 of 512).
constexpr int kWant = 512, kMinKeys = 128;
constexpr int kMostSplits = 256;

KaPlan ka_plan(int64_t R, int64_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  KaPlan pl{};
  pl.tiles = (int)ceil_div(Hq / Hkv, 16);
  const int waves = ka_waves(D <= 64 ? 64 : D <= 128 ? 128 : 256);
  pl.heads = Hkv % waves == 0 ? waves : Hkv % 2 == 0 ? 2 : 1;
  const int64_t units = R * pl.tiles * (Hkv / pl.heads);
  const int64_t most = std::min<int64_t>(ceil_div(S, kMinKeys), kMostSplits);
  pl.splits = (int)std::min(most, ceil_div(kWant, units));
  pl.blocks = ceil_div(R * pl.tiles * pl.splits, 8) * 8 * (Hkv / pl.heads);
  // splits R rows are at most R + kWant heads / (Hkv tiles) rows: `total` never falls as a
  // call grows
  const int64_t rows =
      most == 1 ? 0 : std::min(R * most, R + (int64_t)kWant * pl.heads / (Hkv * pl.tiles)) * Hq;
  pl.ml = align_up((size_t)rows * D * 4, 256);
  pl.total = align_up(pl.ml + (size_t)rows * 8, 256);
  return pl;
}

bool ka_ok(int64_t R, int64_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  return R >= 1 && S >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && D >= 1;
}
bool ka_supported(int64_t R, int64_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  const int64_t lim = (int64_t)1 << 31;
  return D % 32 == 0 && D <= 256 && R < lim / Hq && S < lim && Hkv < (1 << 24) / D &&
         (double)R * Hkv * (double)ceil_div(Hq / Hkv, 16) < (1 << 22);
}

template <typename Tv, int DP, int EACH>
int ka_launch(const KaArgs& a, const KaPlan& pl, hipStream_t st) {
  ka_kernel<Tv, DP, EACH><<<dim3((unsigned)pl.blocks), dim3(64 * ka_waves(DP)), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv>
int ka_run(const KaArgs& a, const KaPlan& pl, hipStream_t st) {
  const int nb = a.D / 32;
  const int rc = nb == 1 ? ka_launch<Tv, 64, 1>(a, pl, st)
               : nb == 2 ? ka_launch<Tv, 64, 2>(a, pl, st)
               : nb == 3 ? ka_launch<Tv, 128, 1>(a, pl, st)
               : nb == 4 ? ka_launch<Tv, 128, 4>(a, pl, st)
               : nb == 6 ? ka_launch<Tv, 256, 2>(a, pl, st)
               : nb == 8 ? ka_launch<Tv, 256, 4>(a, pl, st)
                         : ka_launch<Tv, 256, 1>(a, pl, st);
  if (rc != MOE_OK || a.splits == 1) return rc;
  const JoinArgs jn = {a.part_o, a.part_ml, nullptr, 0, a.R * a.Hq, a.Hq, a.D, a.splits, a.out,
                       a.lse};
  return attention_join<Tv>(jn, st);
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_kv4_attention_workspace(int64_t R, int64_t S, int32_t Hq, int32_t Hkv,
                                              int32_t D) {
  using namespace moe;
  if (!ka_ok(R, S, Hq, Hkv, D) || !ka_supported(R, S, Hq, Hkv, D)) return 0;
  return ka_plan(R, S, Hq, Hkv, D).total;
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
  if ((reinterpret_cast<uintptr_t>(k_scales) | reinterpret_cast<uintptr_t>(v_scales)) & 3)
    return MOE_ERR_UNSUPPORTED;                  // a word of them at a time
  const KaPlan pl = ka_plan(R, S, Hq, Hkv, D);
  const int64_t elt = dtype == MOE_BF16 ? 2 : 4, vals = C * S * Hkv * D;
  const Span in[] = {{q, R * Hq * D * elt}, {k_codes, vals / 2}, {k_scales, vals / 32},
                     {v_codes, vals / 2}, {v_scales, vals / 32}, {cache_row, R * 4}, {lens, R * 4}};
  const Span outs[] = {{out, R * Hq * D * elt}, {lse, R * Hq * 4},
                       {workspace, pl.splits > 1 ? (int64_t)pl.total : 0}};
  MOE_CHECK_ARG(spans_apart(outs, in));
  if (pl.splits > 1 &&
      (!workspace || ws_bytes < pl.total || (reinterpret_cast<uintptr_t>(workspace) & 255)))
    return MOE_ERR_WORKSPACE;
  const ScoreScale sc = score_scale(scale, dtype == MOE_BF16);
  KaArgs a{};
  a.q = q;
  a.codes[0] = k_codes;
  a.codes[1] = v_codes;
  a.scales[0] = k_scales;
  a.scales[1] = v_scales;
  a.cache_row = cache_row;
  a.lens = lens;
  a.R = R;
  a.C = C;
  a.S = S;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.D = D;
  a.nq = Hq / Hkv;
  a.tiles = pl.tiles;
  a.heads = pl.heads;
  a.scale2 = sc.scale2;
  a.keep = sc.keep;
  a.flip = sc.flip;
  a.splits = pl.splits;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + pl.ml);
  a.out = out;
  a.lse = lse;
  hipStream_t st = as_stream(stream);
  return dtype == MOE_BF16 ? ka_run<uint16_t>(a, pl, st) : ka_run<float>(a, pl, st);
}
