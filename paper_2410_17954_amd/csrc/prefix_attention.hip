// moe_prefix_attention: one new token per row; the rows of a group share a
// prefix of keys and values, each row has a suffix of its own.
//
// Bound by reading the caches once (HBM) while a group's query rows are few.
// Computed row by row the prefix would be read once per row; here the queries
// of all rows of a group that read one key head (rows x query heads of it) are
// the columns of the products, so a key is loaded once for all of them.
//   S^T = K Q^T     rows: keys, columns: queries
//   O^T = V^T P^T   rows: values' dimensions, columns: queries
// Transposed so, a lane of the MFMA result holds scores of one query for four
// neighbouring keys: the running maximum and sum are one register each, the
// rescaling of O is lane by lane, and the scores of two 16-key tiles are, in
// place, a lane's eight operands of the second product (its k slots 8q + j are
// keys 4q + j of the first tile and 4q + j - 4 of the second). V^T comes from LDS
// through the transposing read, four keys of one column at a time.
// Waves of a block take 32 keys (16 in float32) at a time in turn and keep a
// maximum, sum and O of their own, so there is no barrier in the loop; they are
// added up through LDS at the end. Long key ranges are split over blocks, and a
// second launch joins the splits of prefix and suffix.
#include "moeflow_decode.h"
#include "common.h"
#include "buffers.h"

#include <math.h>

#include <algorithm>

namespace moe {
namespace {

constexpr int kPaThreads = 256, kPaWaves = kPaThreads / kWave;
constexpr uint32_t kPastEnd = 0x7ffffff0u;       // no buffer here is as long
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PaArgs {
  const void *q, *k_prefix, *v_prefix, *k_suffix, *v_suffix;
  const int32_t *group_offsets, *prefix_len, *suffix_len;
  int64_t R, G, P, S;
  int Hq, Hkv, D, nq;                            // nq: query heads of a key head
  float scale2;                                  // scale * log2 e
  int splits_p, splits_s;                        // of a prefix, of a suffix
  int64_t blocks_p;                              // blocks of the prefixes, which come first
  int64_t slots_p;                               // row tiles of the prefixes (upper bound)
  int tiles_s;                                   // row tiles of a suffix
  float* part_o;                                 // [splits_p + splits_s][R * Hq][D]
  float2* part_ml;                               // [splits_p + splits_s][R * Hq]: max (log2), sum
};

__device__ __forceinline__ int64_t group_row(const PaArgs& a, int64_t g) {
  if (!a.group_offsets) return g * (a.R / a.G);
  return min(max((int64_t)a.group_offsets[g], (int64_t)0), a.R);
}

// What a block works on: `m_n` query columns from m0 on (column m is row
// row0 + m / nq, query head h * nq + m % nq), keys [lo, hi) of a cache.
struct PaJob {
  const char *k, *v;                             // of key 0, head h
  int64_t lo, hi, row0;
  int m0, m_n, h, split;
};

// Row tiles of group g start at slot floor(first row * nq / BM) + g: slots of
// different groups never meet, and a slot's group is found without a scan.
template <typename Tv, int BM>
__device__ __forceinline__ bool find_job(const PaArgs& a, int64_t block, PaJob& j) {
  int64_t len;
  if (block < a.blocks_p) {
    // slots of one head and split are neighbours eight apart: blocks of one
    // XCD share the keys they read in its L2
    const int64_t slot = block / 8 % a.slots_p;
    const int64_t hs = block / (8 * a.slots_p) * 8 + block % 8;
    if (hs >= (int64_t)a.Hkv * a.splits_p) return false;
    j.h = (int)(hs % a.Hkv);
    j.split = (int)(hs / a.Hkv);
    int64_t lo = 0, hi = a.G;                    // last group whose first slot is <= slot
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) / 2;
      if (group_row(a, mid) * a.nq / BM + mid <= slot) lo = mid;
      else hi = mid;
    }
    const int64_t r0 = group_row(a, lo), r1 = group_row(a, lo + 1);
    const int64_t first = r0 * a.nq / BM + lo;
    const int64_t cols = (r1 - r0) * a.nq;
    if (slot < first || (slot - first) * BM >= cols) return false;
    j.row0 = r0;
    j.m0 = (int)((slot - first) * BM);
    j.m_n = (int)min(cols - j.m0, (int64_t)BM);
    const int64_t at = (lo * a.P * a.Hkv + j.h) * a.D;
    j.k = reinterpret_cast<const char*>(static_cast<const Tv*>(a.k_prefix) + at);
    j.v = reinterpret_cast<const char*>(static_cast<const Tv*>(a.v_prefix) + at);
    len = a.prefix_len ? min(max((int64_t)a.prefix_len[lo], (int64_t)0), a.P) : a.P;
    const int64_t per = ((len + a.splits_p - 1) / a.splits_p + 31) / 32 * 32;
    j.lo = min(len, per * j.split);
    j.hi = min(len, j.lo + per);
    return true;
  }
  block -= a.blocks_p;
  j.split = (int)(block % a.splits_s);
  block /= a.splits_s;
  j.h = (int)(block % a.Hkv);
  block /= a.Hkv;
  const int tile = (int)(block % a.tiles_s);
  j.row0 = block / a.tiles_s;
  if (j.row0 >= a.R || j.row0 < group_row(a, 0) || j.row0 >= group_row(a, a.G)) return false;
  j.m0 = tile * 16;
  j.m_n = min(a.nq - j.m0, 16);
  const int64_t at = (j.row0 * a.S * a.Hkv + j.h) * a.D;
  j.k = reinterpret_cast<const char*>(static_cast<const Tv*>(a.k_suffix) + at);
  j.v = reinterpret_cast<const char*>(static_cast<const Tv*>(a.v_suffix) + at);
  len = a.suffix_len ? min(max((int64_t)a.suffix_len[j.row0], (int64_t)0), a.S) : a.S;
  const int64_t per = ((len + a.splits_s - 1) / a.splits_s + 31) / 32 * 32;
  j.lo = min(len, per * j.split);
  j.hi = min(len, j.lo + per);
  j.split += a.splits_p;
  return true;
}

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

// One step of a wave: KT tiles of 16 keys. DP: the dimension padded to whole
// lines of 128 bytes; 16-byte chunks past D are zeros. Rows are loaded as 8 keys
// x 128 bytes an instruction and become MFMA operands by a swap between lanes l
// and l ^ 8 (ror8_into): operand 2l + h of lane (key r, q) holds the line's chunk
// 4h + q.
template <typename Tv, int DP>
struct PaCore {
  static constexpr bool BF16 = sizeof(Tv) == 2;
  static constexpr int KT = BF16 ? 2 : 1, KEYS = 16 * KT;
  static constexpr int VE = 16 / sizeof(Tv);     // values per chunk
  static constexpr int LN = DP * (int)sizeof(Tv) / 128, CHUNKS = 8 * LN;
  static constexpr int QR = 2 * LN;              // operands of a query
  static constexpr int DT = DP / 16;             // 16-dimension tiles of O
  static constexpr int kStage = KEYS * DP * (int)sizeof(Tv);   // bytes of staged values
  struct Rows { u32x4_t v[KEYS / 8][LN]; };

  static __device__ __forceinline__ void load(Rows& r, const char* base, int64_t key, int64_t end,
                                              uint32_t stride, int D) {
    // keys past the end lie past the end of the buffer: zeros
    const int64_t n = min(end - key, (int64_t)KEYS);
    const rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(base + key * stride), 0,
        (int)((uint32_t)(n - 1) * stride + (uint32_t)D * sizeof(Tv)), 0x00027000);
    const int lane = lane_id();
    const int c = (lane >> 4) + ((lane >> 3) & 1) * 4;
#pragma unroll
    for (int g = 0; g < KEYS / 8; ++g)
#pragma unroll
      for (int l = 0; l < LN; ++l) {
        const uint32_t off = (uint32_t)(g * 8 + (lane & 7)) * stride + (l * 8 + c) * 16;
        r.v[g][l] = buf_load16<false>(rs, (l * 8 + c) * VE < D ? off : kPastEnd, 0);
      }
  }
  static __device__ __forceinline__ void mfma(f32x4_t& c, const u32x4_t& x, const u32x4_t& y) {
    if constexpr (BF16) {
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x),
                                                  __builtin_bit_cast(bf16x8_t, y), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[v]), __uint_as_float(y[v]), c,
                                                 0, 0, 0);
    }
  }
  template <int MT>
  static __device__ __forceinline__ void scores(f32x4_t (&s)[MT][KT], const u32x4_t (&q)[MT][QR],
                                                const Rows& k) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) s[i][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int l = 0; l < LN; ++l) {
        u32x4_t k0, k1;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          k0[v] = ror8_into(k.v[2 * kt][l][v], k.v[2 * kt + 1][l][v], true);
          k1[v] = ror8_into(k.v[2 * kt + 1][l][v], k.v[2 * kt][l][v], false);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          mfma(s[i][kt], k0, q[i][2 * l]);
          mfma(s[i][kt], k1, q[i][2 * l + 1]);
        }
      }
  }

  // Staged rows keep their chunks, XORed so that the reads of a tile of O meet
  // different banks: eight rows x 32 bytes (bf16), four rows x 64 (float32).
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (!BF16) return 4 * ((row >> 2) & 3);
    return DP == 64 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
  }
  static __device__ __forceinline__ void stage(char* lds, const Rows& r) {
    const int lane = lane_id();
    const int c = (lane >> 4) + ((lane >> 3) & 1) * 4;
#pragma unroll
    for (int g = 0; g < KEYS / 8; ++g)
#pragma unroll
      for (int l = 0; l < LN; ++l) {
        const int row = g * 8 + (lane & 7);
        *reinterpret_cast<u32x4_t*>(lds + (row * CHUNKS + ((l * 8 + c) ^ swz(row))) * 16) = r.v[g][l];
      }
  }
  // O += V^T P^T
  template <int MT>
  static __device__ __forceinline__ void values(f32x4_t (&o)[MT][DT], const f32x4_t (&p)[MT][KT],
                                                const char* lds) {
    const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
    if constexpr (BF16) {
      // p is rounded to bf16 (at most 2^-9 of it, for the matrix cores); its
      // sum is taken of the float32 values
      bf16x8_t pb[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) pb[i][j] = (__bf16)p[i][j / 4][j % 4];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        s16x4_t v[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const int row = 16 * kt + 4 * q4 + (r >> 2);
          const int c = (2 * dt + ((r >> 1) & 1)) ^ swz(row);
          v[kt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4_t*)(lds + (row * CHUNKS + c) * 16 + (r & 1) * 8));
        }
        const bf16x8_t vt = __builtin_bit_cast(
            bf16x8_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int i = 0; i < MT; ++i)
          o[i][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pb[i], o[i][dt], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int row = 4 * q4 + v;
          const int c = (4 * dt + (r >> 2)) ^ swz(row);
          const float x = *reinterpret_cast<const float*>(lds + (row * CHUNKS + c) * 16 + (r & 3) * 4);
#pragma unroll
          for (int i = 0; i < MT; ++i)
            o[i][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, p[i][0][v], o[i][dt], 0, 0, 0);
        }
    }
  }
};

__device__ __forceinline__ void lds_fence() {    // LDS of one wave: program order is enough
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

template <typename Tv, int DP, int MT>
__device__ __forceinline__ void pa_block(const PaArgs& a, const PaJob& j, char* lds,
                                         float (*s_m)[64], float (*s_l)[64]) {
  using C = PaCore<Tv, DP>;
  constexpr int KT = C::KT, DT = C::DT;
  const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t RH = a.R * a.Hq;
  auto rowhead = [&](int m) {
    return (j.row0 + (j.m0 + m) / a.nq) * a.Hq + j.h * a.nq + (j.m0 + m) % a.nq;
  };
  if (j.lo >= j.hi) {                            // no keys: this split adds nothing
    for (int m = threadIdx.x; m < j.m_n; m += kPaThreads)
      a.part_ml[j.split * RH + rowhead(m)] = make_float2(-INFINITY, 0.f);
    return;
  }
  u32x4_t q[MT][C::QR];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = 16 * i + r;
    const Tv* const qr = static_cast<const Tv*>(a.q) + (m < j.m_n ? rowhead(m) : 0) * a.D;
#pragma unroll
    for (int s = 0; s < C::QR; ++s) {
      const int d = (4 * s + q4) * C::VE;
      q[i][s] = m < j.m_n && d < a.D ? *reinterpret_cast<const u32x4_t*>(qr + d) : u32x4_t{0, 0, 0, 0};
    }
  }
  f32x4_t o[MT][DT];
  float m_run[MT], l_run[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[i][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  char* const mine = lds + wave * C::kStage;
  const uint32_t stride = (uint32_t)(a.Hkv * a.D * (int)sizeof(Tv));
  typename C::Rows k, v;
  int64_t key = j.lo + wave * C::KEYS;
  if (key < j.hi) {
    C::load(k, j.k, key, j.hi, stride, a.D);
    C::load(v, j.v, key, j.hi, stride, a.D);
  }
  while (key < j.hi) {
    f32x4_t s[MT][KT];
    C::template scores<MT>(s, q, k);
    C::stage(mine, v);
    const int64_t next = key + kPaWaves * C::KEYS;
    if (next < j.hi) {
      C::load(k, j.k, next, j.hi, stride, a.D);
      C::load(v, j.v, next, j.hi, stride, a.D);
    }
    const bool ragged = key + C::KEYS > j.hi;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float t = s[i][kt][e] * a.scale2;
          if (ragged && key + 16 * kt + 4 * q4 + e >= j.hi) t = -INFINITY;
          s[i][kt][e] = t;
          mx = fmaxf(mx, t);
        }
      mx = fmaxf(m_run[i], quad_max(mx));
      const float mu = mx == -INFINITY ? 0.f : mx;         // nothing but -inf so far
      if (ballot(mx > m_run[i])) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[i] - mu);
        l_run[i] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[i][dt] *= alpha;
        m_run[i] = mx;
      }
      float sum = 0.f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[i][kt][e] = __builtin_amdgcn_exp2f(s[i][kt][e] - mu);
          sum += s[i][kt][e];
        }
      l_run[i] += sum;
    }
    lds_fence();
    C::template values<MT>(o, s, mine);
    lds_fence();
    key = next;
  }
  // join the waves: common maximum, then O through LDS, one row tile at a time
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const float l = quad_sum(l_run[i]);
    if (q4 == 0) {
      s_m[wave][16 * i + r] = m_run[i];
      s_l[wave][16 * i + r] = l;
    }
  }
  __syncthreads();                               // and every wave is done with its stage
  f32x4_t* const part = reinterpret_cast<f32x4_t*>(lds);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = 16 * i + r;
    float top = s_m[0][m];
#pragma unroll
    for (int w = 1; w < kPaWaves; ++w) top = fmaxf(top, s_m[w][m]);
    const float mu = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m_run[i] - mu);
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kPaWaves; ++w) l += s_l[w][m] * __builtin_amdgcn_exp2f(s_m[w][m] - mu);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) part[(wave * DT + dt) * kWave + lane] = o[i][dt] * f;
    __syncthreads();
    if (m < j.m_n) {
      const int64_t at = j.split * RH + rowhead(m);
      if (wave == 0 && q4 == 0) a.part_ml[at] = make_float2(top, l);
#pragma unroll
      for (int t = 0; t < DT / kPaWaves; ++t) {
        const int dt = wave * (DT / kPaWaves) + t;
        f32x4_t sum = part[dt * kWave + lane];
#pragma unroll
        for (int w = 1; w < kPaWaves; ++w) sum += part[(w * DT + dt) * kWave + lane];
        const int d = 16 * dt + 4 * q4;          // D is a multiple of 8
        if (d < a.D) *reinterpret_cast<f32x4_t*>(a.part_o + at * a.D + d) = sum;
      }
    }
    __syncthreads();                             // part is rewritten next
  }
}

// MT: 16-column tiles of a prefix block; suffix blocks have one. The most that
// leaves every instance without a spilled register; with four, or dimensions
// past 128, one wave a SIMD has all of them.
constexpr int pa_max_tiles(int elt, int dp) {
  return dp == 256 ? 1 : dp == 128 && elt == 4 ? 2 : 4;
}
template <typename Tv, int DP, int MT>
__global__ void __launch_bounds__(kPaThreads, MT == 4 || DP == 256 ? 1 : 2)
pa_kernel(PaArgs a) {
  using C = PaCore<Tv, DP>;
  __shared__ __attribute__((aligned(16))) char lds[kPaWaves * C::kStage];
  __shared__ float s_m[kPaWaves][64], s_l[kPaWaves][64];
  static_assert(kPaWaves * C::kStage >= kPaWaves * C::DT * kWave * 16, "O of the waves");
  PaJob j;
  if (!find_job<Tv, 16 * MT>(a, blockIdx.x, j)) return;
  if ((int64_t)blockIdx.x < a.blocks_p) pa_block<Tv, DP, MT>(a, j, lds, s_m, s_l);
  else pa_block<Tv, DP, 1>(a, j, lds, s_m, s_l);
}

// Row r, head h: the splits' O, sums and maxima joined. tpr threads (a power of
// two, at least D / 4) a row and head.
template <typename Tv>
__global__ void __launch_bounds__(kPaThreads)
pa_join_kernel(PaArgs a, int tpr_shift, Tv* __restrict__ out, float* __restrict__ lse) {
  const int64_t RH = a.R * a.Hq;
  const int64_t at = ((int64_t)blockIdx.x * kPaThreads + threadIdx.x) >> tpr_shift;
  const int d = 4 * (threadIdx.x & ((1 << tpr_shift) - 1));
  if (at >= RH || d >= a.D) return;
  const int64_t row = at / a.Hq;
  if (row < group_row(a, 0) || row >= group_row(a, a.G)) return;
  const int n = a.splits_p + a.splits_s;
  float m = -INFINITY;
  for (int p = 0; p < n; ++p) m = fmaxf(m, a.part_ml[p * RH + at].x);
  const float mu = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < n; ++p) {
    const float2 ml = a.part_ml[p * RH + at];
    if (ml.y == 0.f) continue;                   // a split without keys wrote no O
    const float f = __builtin_amdgcn_exp2f(ml.x - mu);
    l += ml.y * f;
    o += *reinterpret_cast<const f32x4_t*>(a.part_o + (p * RH + at) * a.D + d) * f;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  Tv* const dst = out + at * a.D + d;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(Tv) == 2) dst[e] = f32_to_bf16(o[e] * inv);
    else dst[e] = o[e] * inv;
  }
  if (lse && d == 0) lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

struct PaPlan {
  int mt, dp, splits_p, splits_s, tiles_s;
  int64_t slots_p, blocks_p, blocks_s;
  size_t o, ml, total;
};

PaPlan pa_plan(int64_t R, int64_t G, int32_t Hq, int32_t Hkv, int32_t D, int64_t P, int64_t S,
               int32_t dtype) {
  PaPlan pl{};
  const int nq = Hq / Hkv;
  pl.dp = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  const int64_t cols = ceil_div(R, G) * nq;      // of an average group
  pl.mt = std::min(cols <= 16 ? 1 : cols <= 32 ? 2 : 4,
                   pa_max_tiles(dtype == MOE_BF16 ? 2 : 4, pl.dp));
  pl.slots_p = R * nq / (16 * pl.mt) + G;
  pl.tiles_s = (int)ceil_div(nq, 16);
  auto splits = [](int64_t blocks, int64_t keys) {
    if (keys == 0) return 0;
    const int64_t most = std::min<int64_t>(ceil_div(keys, 128), 64);
    return (int)std::min(most, std::max<int64_t>(1, ceil_div(512, blocks)));
  };
  // the tiles of even groups; the upper bound counts one more a group
  const int64_t used = G * ceil_div(cols, 16 * pl.mt);
  pl.splits_p = splits(used * Hkv, P);
  pl.splits_s = splits(R * Hkv * pl.tiles_s, S);
  pl.blocks_p = pl.splits_p ? ceil_div((int64_t)Hkv * pl.splits_p, 8) * 8 * pl.slots_p : 0;
  pl.blocks_s = R * Hkv * pl.tiles_s * pl.splits_s;
  const size_t n = (size_t)(pl.splits_p + pl.splits_s) * R * Hq;
  pl.o = 0;
  pl.ml = align_up(n * D * 4, 256);
  pl.total = align_up(pl.ml + n * 8, 256);
  return pl;
}

bool pa_ok(int64_t R, int64_t G, int32_t Hq, int32_t Hkv, int32_t D, int64_t P, int64_t S,
           int32_t dtype) {
  return R >= 1 && G >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && D >= 1 && P >= 0 && S >= 0 &&
         valid_dtype(dtype);
}
bool pa_supported(int64_t R, int64_t G, int32_t Hq, int32_t Hkv, int32_t D, int64_t P, int64_t S,
                  int32_t dtype) {
  const int64_t elt = dtype == MOE_BF16 ? 2 : 4, lim = (int64_t)1 << 31;
  if (D % 8 || D > 256 || G > R || P >= lim || S >= lim) return false;
  if (R >= lim / Hq || (int64_t)Hkv >= lim / (32 * elt * D)) return false;
  if ((double)G * (double)P * Hkv * D * elt > 4e18 || (double)R * (double)S * Hkv * D * elt > 4e18)
    return false;
  const PaPlan pl = pa_plan(R, G, Hq, Hkv, D, P, S, dtype);
  return pl.blocks_p + pl.blocks_s < lim && ceil_div(R * Hq, 4) < lim;
}

template <typename Tv, int DP>
int pa_launch(const PaArgs& a, int mt, unsigned blocks, hipStream_t st) {
  constexpr int M = pa_max_tiles(sizeof(Tv), DP);
  if (mt == 1) pa_kernel<Tv, DP, 1><<<dim3(blocks), dim3(kPaThreads), 0, st>>>(a);
  if constexpr (M >= 2)
    if (mt == 2) pa_kernel<Tv, DP, 2><<<dim3(blocks), dim3(kPaThreads), 0, st>>>(a);
  if constexpr (M >= 4)
    if (mt == 4) pa_kernel<Tv, DP, 4><<<dim3(blocks), dim3(kPaThreads), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv>
int pa_run(const PaArgs& a, const PaPlan& pl, Tv* out, float* lse, hipStream_t st) {
  const unsigned blocks = (unsigned)(pl.blocks_p + pl.blocks_s);
  int rc = MOE_OK;
  if (blocks) {
    rc = pl.dp == 64 ? pa_launch<Tv, 64>(a, pl.mt, blocks, st)
       : pl.dp == 128 ? pa_launch<Tv, 128>(a, pl.mt, blocks, st)
                      : pa_launch<Tv, 256>(a, pl.mt, blocks, st);
  }
  if (rc != MOE_OK) return rc;
  const int shift = a.D <= 64 ? 4 : a.D <= 128 ? 5 : 6;
  const unsigned grid = (unsigned)ceil_div(a.R * a.Hq, kPaThreads >> shift);
  pa_join_kernel<Tv><<<dim3(grid), dim3(kPaThreads), 0, st>>>(a, shift, out, lse);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_prefix_attention_workspace(int64_t R, int64_t G, int32_t Hq, int32_t Hkv,
                                                 int32_t D, int64_t P, int64_t S, int32_t dtype) {
  using namespace moe;
  if (!pa_ok(R, G, Hq, Hkv, D, P, S, dtype) || !pa_supported(R, G, Hq, Hkv, D, P, S, dtype))
    return 0;
  return pa_plan(R, G, Hq, Hkv, D, P, S, dtype).total;
}

extern "C" int moe_prefix_attention(const void* q, int32_t dtype, int64_t R, int32_t Hq,
                                    int32_t Hkv, int32_t D, const int32_t* group_offsets, int64_t G,
                                    const void* k_prefix, const void* v_prefix, int64_t P,
                                    const int32_t* prefix_len, const void* k_suffix,
                                    const void* v_suffix, int64_t S, const int32_t* suffix_len,
                                    float scale, void* out, float* lse, void* workspace,
                                    size_t ws_bytes, void* stream) {
  using namespace moe;
  MOE_CHECK_ARG(q && out && pa_ok(R, G, Hq, Hkv, D, P, S, dtype));
  MOE_CHECK_ARG((P == 0 || (k_prefix && v_prefix)) && (S == 0 || (k_suffix && v_suffix)));
  MOE_CHECK_ARG(group_offsets || R % G == 0);
  MOE_CHECK_ARG(isfinite(scale));
  if (!pa_supported(R, G, Hq, Hkv, D, P, S, dtype)) return MOE_ERR_UNSUPPORTED;
  uintptr_t bits = 0;
  for (const void* p : {q, k_prefix, v_prefix, k_suffix, v_suffix, static_cast<const void*>(out)})
    bits |= reinterpret_cast<uintptr_t>(p);
  if (bits & 15) return MOE_ERR_UNSUPPORTED;     // 16-byte loads
  const PaPlan pl = pa_plan(R, G, Hq, Hkv, D, P, S, dtype);
  if (pl.total && (!workspace || ws_bytes < pl.total || (reinterpret_cast<uintptr_t>(workspace) & 255)))
    return MOE_ERR_WORKSPACE;
  char* const ws = static_cast<char*>(workspace);
  PaArgs a{};
  a.q = q;
  a.k_prefix = k_prefix;
  a.v_prefix = v_prefix;
  a.k_suffix = k_suffix;
  a.v_suffix = v_suffix;
  a.group_offsets = group_offsets;
  a.prefix_len = prefix_len;
  a.suffix_len = suffix_len;
  a.R = R;
  a.G = G;
  a.P = P;
  a.S = S;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.D = D;
  a.nq = Hq / Hkv;
  a.scale2 = scale * kLog2e;
  a.splits_p = pl.splits_p;
  a.splits_s = pl.splits_s;
  a.blocks_p = pl.blocks_p;
  a.slots_p = pl.slots_p;
  a.tiles_s = pl.tiles_s;
  a.part_o = reinterpret_cast<float*>(ws + pl.o);
  a.part_ml = reinterpret_cast<float2*>(ws + pl.ml);
  hipStream_t st = as_stream(stream);
  return dtype == MOE_BF16 ? pa_run<uint16_t>(a, pl, static_cast<uint16_t*>(out), lse, st)
                           : pa_run<float>(a, pl, static_cast<float*>(out), lse, st);
}
