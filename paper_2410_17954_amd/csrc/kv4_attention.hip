// moe_kv4_attention: single tokens over a cache in 4 bits.
//
// Bound by reading the cache once (HBM): 17/32 byte a value. A block takes one row, one
// key head (its query heads are the columns of the products) and a range of keys:
//   S^T = K Q^T     rows: keys, columns: queries
//   O^T = V^T P^T   rows: values' dimensions, columns: queries
// Codes become bf16 in registers, two an instruction with their block's scale: exact,
// as each value is a number of two bits times a power of two. A lane holds a quarter
// of a key's head, whole blocks or halves of one, so keys are MFMA operands as they
// were loaded (k slots 8t + j of quarter q4 are dimensions q4 D/4 + 8t + j, of the
// queries too); values are staged in LDS and come back through the transposing read.
// float32 queries and numerators are cut into three bf16 numbers of 8 bits each,
// whose products are exact: three MFMAs for one, which the cache's stream hides.
// Waves of a block take 32 keys at a time in turn, the next ones' codes in flight, and
// keep a maximum, sum and O of their own; they are added up through LDS at the end.
// Long key ranges are split over blocks, and a second launch joins the splits.
#include "moeflow_prompt.h"
#include "attention.h"
#include "buffers.h"
#include "spans.h"

#include <algorithm>

namespace moe {
namespace {

constexpr int KEYS = 32, KT = 2;                 // of a wave's step
constexpr uint32_t kPastEnd = 0x7ffffff0u;       // no buffer here is as long

struct KaArgs {
  const void* q;
  const uint8_t *codes[2], *scales[2];           // of keys, of values
  const int32_t *cache_row, *lens;
  int64_t R, C, S;
  int Hq, Hkv, D, nq, tiles;                     // tiles: of 16 query heads of a key head
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

// x as a sum of NS bf16 numbers: cut, not rounded, so that three hold all 24 bits.
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

// DP: the dimension padded to 64, 128 or 256; channels past D are zeros.
template <typename Tv, int DP>
struct KaCore {
  static constexpr bool BF16 = sizeof(Tv) == 2;
  static constexpr int NS = BF16 ? 1 : 3;        // bf16 numbers of a query's channel
  static constexpr int WN = DP / 32;             // words of a lane's quarter, QK k-steps
  static constexpr int SN = DP == 256 ? 2 : 1;   // scales of a lane's quarter
  static constexpr int DT = DP / 16, CH = DP / 8;
  static constexpr int kStage = KEYS * DP * 2;
  struct Codes { uint32_t w[KT][WN]; uint8_t s[KT][SN]; };

  static __device__ __forceinline__ void load(Codes& x, const uint8_t* codes, const uint8_t* scales,
                                              int64_t key, int64_t end, const KaArgs& a) {
    // keys past the end lie past the end of the buffers: zeros
    const int n = (int)min(end - key, (int64_t)KEYS);
    const uint32_t row = (uint32_t)(a.Hkv * (a.D / 2)), srow = (uint32_t)(a.Hkv * (a.D / 32));
    const rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(codes + key * row), 0, (int)((n - 1) * row + a.D / 2), 0x00027000);
    const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(scales + key * srow), 0, (int)((n - 1) * srow + a.D / 32), 0x00027000);
    const int r = lane_id() & 15, q4 = lane_id() >> 4;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const uint32_t k = 16 * kt + r;
      if constexpr (DP == 64) {
        const uint32_t off = q4 * 8 < a.D / 2 ? k * row + q4 * 8 : kPastEnd;
        const u32x2_t w = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rc, (int)off, 0, 2));
        x.w[kt][0] = w[0];
        x.w[kt][1] = w[1];
      } else {
#pragma unroll
        for (int i = 0; i < WN / 4; ++i) {
          const int at = q4 * (DP / 8) + 16 * i;
          const u32x4_t w = buf_load16<true>(rc, at < a.D / 2 ? k * row + at : kPastEnd, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e) x.w[kt][4 * i + e] = w[e];
        }
      }
#pragma unroll
      for (int i = 0; i < SN; ++i) {
        const int at = DP == 64 ? q4 / 2 : SN * q4 + i;
        x.s[kt][i] = __builtin_amdgcn_raw_buffer_load_b8(
            rs, (int)(at < a.D / 32 ? k * srow + at : kPastEnd), 0, 0);
      }
    }
  }
  static __device__ __forceinline__ float scale_of(const Codes& x, int kt, int t) {
    return __uint_as_float((uint32_t)x.s[kt][SN == 2 ? t / 4 : 0] << 23);
  }
  static __device__ __forceinline__ void scores(f32x4_t (&s)[1][KT], const u32x4_t (&q)[NS][WN],
                                                const Codes& k) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) s[0][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < WN; ++t)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const u32x4_t x = eight_bf16(k.w[kt][t], scale_of(k, kt, t));
#pragma unroll
        for (int n = 0; n < NS; ++n) mfma(s[0][kt], x, q[n][t]);
      }
  }
  // Staged rows keep their 16-byte chunks, XORed so that reads and writes of sixteen
  // rows meet different banks.
  static __device__ __forceinline__ int swz(int row) {
    return DP == 64 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
  }
  static __device__ __forceinline__ void stage(char* lds, const Codes& v) {
    const int r = lane_id() & 15, q4 = lane_id() >> 4;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int t = 0; t < WN; ++t)
        *reinterpret_cast<u32x4_t*>(lds + ((16 * kt + r) * CH + ((q4 * WN + t) ^ swz(r))) * 16) =
            eight_bf16(v.w[kt][t], scale_of(v, kt, t));
  }
  // O += V^T P^T. bf16: p is rounded to bf16 (at most 2^-8 of it, for the matrix cores);
  // its sum is taken of the float32 values.
  static __device__ __forceinline__ void values(f32x4_t (&o)[1][DT], const f32x4_t (&p)[1][KT],
                                                const char* lds) {
    const int r = lane_id() & 15, q4 = lane_id() >> 4;
    typedef __attribute__((ext_vector_type(8))) uint16_t u16x8_t;
    u32x4_t pb[NS];
    if constexpr (BF16) {
      bf16x8_t b;
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = (__bf16)p[0][j / 4][j % 4];
      pb[0] = __builtin_bit_cast(u32x4_t, b);
    } else {
      u16x8_t b[NS];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint16_t part[NS];
        cut<NS>(p[0][j / 4][j % 4], part);
#pragma unroll
        for (int n = 0; n < NS; ++n) b[n][j] = part[n];
      }
#pragma unroll
      for (int n = 0; n < NS; ++n) pb[n] = __builtin_bit_cast(u32x4_t, b[n]);
    }
    const int row = 4 * q4 + (r >> 2), at = row * CH + (((r >> 1) & 1) ^ swz(row));
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const char* const from = lds + (at ^ (2 * dt)) * 16 + (r & 1) * 8;
      s16x4_t v[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(from + t * 16 * CH * 16));
      const u32x4_t vt = __builtin_bit_cast(
          u32x4_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int n = 0; n < NS; ++n) mfma(o[0][dt], vt, pb[n]);
    }
  }
};

__device__ __forceinline__ void lds_fence() {    // LDS of one wave: program order is enough
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// Waves a SIMD, the most that leave no spilled register.
constexpr int ka_occupancy(int elt, int dp) {
  return dp == 256 ? (elt == 4 ? 1 : 2) : elt == 4 && dp == 128 ? 3 : 4;
}

template <typename Tv, int DP, int W>
__global__ void __launch_bounds__(64 * W, ka_occupancy(sizeof(Tv), DP))
ka_kernel(KaArgs a) {
  using C = KaCore<Tv, DP>;
  constexpr int DT = C::DT;
  __shared__ __attribute__((aligned(16))) char lds[W * C::kStage];
  __shared__ float s_m[W][16], s_l[W][16];
  static_assert(C::kStage >= DT * kWave * 16, "O of the waves");
  // Block b runs on XCD b % 8. Units (row, split, tile) are dealt to the XCDs and an XCD
  // takes all heads of one: heads lie next to each other in a cache, and share its lines.
  const int64_t v = (int64_t)blockIdx.x / (8 * a.Hkv) * 8 + blockIdx.x % 8;
  const int h = (int)(blockIdx.x / 8 % a.Hkv), tile = (int)(v % a.tiles);
  const int split = (int)(v / a.tiles % a.splits);
  const int64_t row = v / a.tiles / a.splits;
  if (row >= a.R) return;
  const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t from = a.cache_row ? (int64_t)a.cache_row[row] : row;
  int64_t len = a.lens ? min(max((int64_t)a.lens[row], (int64_t)0), a.S) : a.S;
  if (from < 0 || from >= a.C) len = 0;
  const int64_t per = ((len + a.splits - 1) / a.splits + KEYS - 1) / KEYS * KEYS;
  const int64_t lo = min(len, per * split), hi = min(len, lo + per);
  const int cols = min(a.nq - tile * 16, 16);
  const int64_t RH = a.R * a.Hq, at = row * a.Hq + h * a.nq + tile * 16 + r, to = split * RH + at;
  if (lo >= hi && a.splits > 1) {                // no keys: this split adds nothing
    if (wave == 0 && q4 == 0 && r < cols) a.part_ml[to] = make_float2(-INFINITY, 0.f);
    return;
  }
  const int64_t base = (from * a.S * a.Hkv + h) * (a.D / 32);   // of the scales; codes 16 a block
  u32x4_t q[C::NS][C::WN];
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
        uint16_t p0[C::NS], p1[C::NS];
        cut<C::NS>(__uint_as_float(x[j / 2][2 * (j % 2)]), p0);
        cut<C::NS>(__uint_as_float(x[j / 2][2 * (j % 2) + 1]), p1);
#pragma unroll
        for (int n = 0; n < C::NS; ++n) q[n][t][j] = (uint32_t)p0[n] | (uint32_t)p1[n] << 16;
      }
    }
  }
  f32x4_t o[1][DT];
  float m_run[1] = {-INFINITY}, l_run[1] = {0.f};
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[0][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  char* const mine = lds + wave * C::kStage;
  const int64_t steps = (hi - lo + KEYS - 1) / KEYS;
  typename C::Codes k, vv;
  auto load = [&](int64_t st) {
    C::load(k, a.codes[0] + base * 16, a.scales[0] + base, lo + st * KEYS, hi, a);
    C::load(vv, a.codes[1] + base * 16, a.scales[1] + base, lo + st * KEYS, hi, a);
  };
  if (wave < steps) load(wave);
  for (int64_t st = wave; st < steps; st += W) {
    f32x4_t s[1][KT];
    C::scores(s, q, k);
    C::stage(mine, vv);
    if (st + W < steps) load(st + W);
    const int keys = (int)min(hi - lo - st * KEYS, (int64_t)KEYS);
    if (keys < KEYS) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * kt + 4 * q4 + e >= keys) s[0][kt][e] = -INFINITY;
    }
    softmax_step(s, m_run, l_run, o, a.scale2);
    lds_fence();
    C::values(o, s, mine);
    lds_fence();
  }
  // join the waves: common maximum, then O through LDS
  const float lw = quad_sum(l_run[0]);
  if (q4 == 0) {
    s_m[wave][r] = m_run[0];
    s_l[wave][r] = lw;
  }
  __syncthreads();                               // and every wave is done with its stage
  f32x4_t* const part = reinterpret_cast<f32x4_t*>(lds);
  float top = s_m[0][r];
#pragma unroll
  for (int w = 1; w < W; ++w) top = fmaxf(top, s_m[w][r]);
  const float mu = top == -INFINITY ? 0.f : top;
  const float f = __builtin_amdgcn_exp2f(m_run[0] - mu);
  float l = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) l += s_l[w][r] * __builtin_amdgcn_exp2f(s_m[w][r] - mu);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) part[(wave * DT + dt) * kWave + lane] = o[0][dt] * f;
  __syncthreads();
  if (r >= cols) return;
  if (wave == 0 && q4 == 0) {
    if (a.splits > 1) a.part_ml[to] = make_float2(top, l);
    else if (a.lse) a.lse[at] = lse_of(top, l);
  }
  for (int dt = wave; dt < DT; dt += W) {
    f32x4_t sum = part[dt * kWave + lane];
#pragma unroll
    for (int w = 1; w < W; ++w) sum += part[(w * DT + dt) * kWave + lane];
    const int d = 16 * dt + 4 * q4;              // D is a multiple of 32
    if (d >= a.D) continue;
    if (a.splits > 1) *reinterpret_cast<f32x4_t*>(a.part_o + to * a.D + d) = sum;
    else put4(static_cast<Tv*>(a.out) + at * a.D + d, sum * (l == 0.f ? 0.f : 1.f / l));
  }
}

struct KaPlan {
  int dp, waves, tiles, splits;
  int64_t blocks;
  size_t ml, total;
};

constexpr int kWant = 1024;                      // blocks that fill the card

KaPlan ka_plan(int64_t R, int64_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  KaPlan pl{};
  pl.dp = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  pl.tiles = (int)ceil_div(Hq / Hkv, 16);
  const int64_t units = R * Hkv * pl.tiles;
  const int64_t most = std::min<int64_t>(ceil_div(S, 256), 128);
  pl.splits = (int)std::min(most, ceil_div(kWant, units));
  pl.waves = pl.splits == 1 && units < 512 ? 8 : 4;
  pl.blocks = ceil_div(R * pl.tiles * pl.splits, 8) * 8 * Hkv;
  // splits R rows are at most R + kWant / (Hkv tiles) rows: `total` never falls as a call
  // grows
  const int64_t rows = most == 1 ? 0 : std::min(R * most, R + kWant / (Hkv * pl.tiles)) * Hq;
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

template <typename Tv, int DP>
int ka_launch(const KaArgs& a, const KaPlan& pl, hipStream_t st) {
  constexpr int W8 = DP == 256 ? 4 : 8;          // stages of 16 KB
  const dim3 grid((unsigned)pl.blocks);
  if (pl.waves == 8) ka_kernel<Tv, DP, W8><<<grid, dim3(64 * W8), 0, st>>>(a);
  else ka_kernel<Tv, DP, 4><<<grid, dim3(64 * 4), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv>
int ka_run(const KaArgs& a, const KaPlan& pl, hipStream_t st) {
  const int rc = pl.dp == 64 ? ka_launch<Tv, 64>(a, pl, st)
               : pl.dp == 128 ? ka_launch<Tv, 128>(a, pl, st)
                              : ka_launch<Tv, 256>(a, pl, st);
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
