// moe_prefix_attention: one new token per row; the rows of a group share a
// prefix of keys and values, each row has a suffix of its own.
//
// Bound by reading the caches once (HBM) while a group's query rows are few.
// Computed row by row the prefix would be read once per row; here the queries
// of all rows of a group that read one key head (rows x query heads of it) are
// the columns of the products, so a key is loaded once for a tile of them: up to 64
// columns, beyond that up to 256 in bfloat16; 16 of D > 128, 32 of float32 with
// D > 64. The tile is that of an average group: larger ones, and more columns than
// the widest tile, read the prefix once a tile.
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
// second launch joins the splits of prefix and suffix; where keys and rows are few, a
// block does a row's prefix and suffix in one launch.
#include "moeflow_decode.h"
#include "common.h"
#include "buffers.h"

#include <math.h>

#include <algorithm>

namespace moe {
namespace {

constexpr int kJoinThreads = 256;
constexpr uint32_t kPastEnd = 0x7ffffff0u;       // no buffer here is as long
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PaArgs {
  const void *q, *k_prefix, *v_prefix, *k_suffix, *v_suffix;
  const int32_t *group_offsets, *prefix_len, *suffix_len;
  int64_t R, G, P, S;
  int Hq, Hkv, D, nq;                            // nq: query heads of a key head
  float scale2;                                  // |scale| log2 e
  uint32_t keep, flip;                           // q & keep ^ flip: no bits where scale is 0,
                                                 // signs turned where it is negative
  int splits_p, splits_s;                        // of a prefix, of a suffix
  int64_t blocks_p;                              // blocks of the prefixes, which come first
  int64_t slots_p;                               // row tiles of the prefixes (upper bound)
  int tiles_s;                                   // row tiles of a suffix
  float* part_o;                                 // [splits_p + splits_s][R * Hq][D]
  float2* part_ml;                               // [splits_p + splits_s][R * Hq]: max (log2), sum
  void* out;
  float* lse;
};

__device__ __forceinline__ int64_t group_row(const PaArgs& a, int64_t g) {
  if (!a.group_offsets) return g * (a.R / a.G);
  return min(max((int64_t)a.group_offsets[g], (int64_t)0), a.R);
}

// What a block works on: `m_n` query columns from m0 on (column m is row
// row0 + m / nq, query head h * nq + m % nq), keys [lo, hi) of a cache and, of a
// whole row, [0, hi2) of another.
struct PaJob {
  const char *k, *v, *k2, *v2;                   // of key 0, head h
  int64_t lo, hi, hi2, row0;
  int m0, m_n, h, split;
};

__device__ __forceinline__ int64_t pa_prefix_len(const PaArgs& a, int64_t g) {
  return a.prefix_len ? min(max((int64_t)a.prefix_len[g], (int64_t)0), a.P) : a.P;
}
__device__ __forceinline__ int64_t pa_suffix_len(const PaArgs& a, int64_t r) {
  return a.suffix_len ? min(max((int64_t)a.suffix_len[r], (int64_t)0), a.S) : a.S;
}

// Row tiles of group g start at slot floor(first row * nq / BM) + g: slots of
// different groups never meet, and a slot's group is found without a scan.
template <typename Tv, int BM>
__device__ __forceinline__ bool find_job(const PaArgs& a, int64_t block, PaJob& j) {
  // Block b runs on XCD b % 8. Units (row tile, split) are dealt to the XCDs and an
  // XCD takes all heads of one: heads lie next to each other in a cache, and an XCD
  // that read one head only would load few channels of its L2 (268 MB of keys and
  // values of 8 heads 73 us, 4 rows).
  int64_t len;
  const bool prefix = block < a.blocks_p;
  if (!prefix) block -= a.blocks_p;
  const int64_t v = block / (8 * a.Hkv) * 8 + block % 8;
  j.h = (int)(block / 8 % a.Hkv);
  if (prefix) {
    const int64_t slot = v / a.splits_p;
    j.split = (int)(v % a.splits_p);
    if (slot >= a.slots_p) return false;
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
    len = pa_prefix_len(a, lo);
    const int64_t per = ((len + a.splits_p - 1) / a.splits_p + 31) / 32 * 32;
    j.lo = min(len, per * j.split);
    j.hi = min(len, j.lo + per);
    return true;
  }
  j.split = (int)(v % a.splits_s);
  const int tile = (int)(v / a.splits_s % a.tiles_s);
  j.row0 = v / a.splits_s / a.tiles_s;
  if (j.row0 >= a.R || j.row0 < group_row(a, 0) || j.row0 >= group_row(a, a.G)) return false;
  j.m0 = tile * 16;
  j.m_n = min(a.nq - j.m0, 16);
  const int64_t at = (j.row0 * a.S * a.Hkv + j.h) * a.D;
  j.k = reinterpret_cast<const char*>(static_cast<const Tv*>(a.k_suffix) + at);
  j.v = reinterpret_cast<const char*>(static_cast<const Tv*>(a.v_suffix) + at);
  len = pa_suffix_len(a, j.row0);
  const int64_t per = ((len + a.splits_s - 1) / a.splits_s + 31) / 32 * 32;
  j.lo = min(len, per * j.split);
  j.hi = min(len, j.lo + per);
  j.split += a.splits_p;
  return true;
}

// Block -> row, key head and column tile of a call that needs no splits.
template <typename Tv>
__device__ __forceinline__ bool find_row(const PaArgs& a, int64_t block, PaJob& j) {
  j.h = (int)(block % a.Hkv);
  j.m0 = (int)(block / a.Hkv % a.tiles_s) * 16;
  j.m_n = min(a.nq - j.m0, 16);
  j.row0 = block / a.Hkv / a.tiles_s;
  int64_t g = 0, end = a.G;                      // last group that starts at or before the row
  while (end - g > 1) {
    const int64_t mid = (g + end) / 2;
    if (group_row(a, mid) <= j.row0) g = mid;
    else end = mid;
  }
  if (j.row0 < group_row(a, g) || j.row0 >= group_row(a, g + 1)) return false;
  const int64_t p = (g * a.P * a.Hkv + j.h) * a.D, s = (j.row0 * a.S * a.Hkv + j.h) * a.D;
  j.k = reinterpret_cast<const char*>(static_cast<const Tv*>(a.k_prefix) + p);
  j.v = reinterpret_cast<const char*>(static_cast<const Tv*>(a.v_prefix) + p);
  j.k2 = reinterpret_cast<const char*>(static_cast<const Tv*>(a.k_suffix) + s);
  j.v2 = reinterpret_cast<const char*>(static_cast<const Tv*>(a.v_suffix) + s);
  j.lo = 0;
  j.hi = pa_prefix_len(a, g);
  j.hi2 = pa_suffix_len(a, j.row0);
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
// x 128 bytes an instruction, non-temporal (a block is mostly the only reader of its
// keys: 4 rows behind 65536 keys 55 us without the hint, 49 with it; four prompts of
// 2000 keys that stay in the caches between calls 13.3, 14.6), and become MFMA
// operands by a swap between lanes l and l ^ 8 (ror8_into): operand 2l + h of lane
// (key r, q) holds the line's chunk 4h + q.
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
        r.v[g][l] = buf_load16<true>(rs, (l * 8 + c) * VE < D ? off : kPastEnd, 0);
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
      // p is rounded to bf16 (at most 2^-8 of it, for the matrix cores); its
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

// Scores -> softmax numerators of one step, in place, for MT column tiles; keys
// from hi - key on are none. m: reference of the numerators 2^(s scale2 - m), raised
// (and l and o rescaled) only where a score exceeds it by more than kSlack, so that
// most steps rescale nothing and numerators stay below 2^kSlack. One branch for all
// tiles: the rest of a step is straight code.
constexpr float kSlack = 8.f;

template <int MT, int KT, int DT>
__device__ __forceinline__ void pa_softmax(f32x4_t (&s)[MT][KT], float (&m)[MT], float (&l)[MT],
                                           f32x4_t (&o)[MT][DT], float scale2, int keys) {
  const int q4 = lane_id() >> 4;
  if (keys < 16 * KT) {                          // scale2 > 0: no weight
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * kt + 4 * q4 + e >= keys) s[i][kt][e] = -INFINITY;
  }
  float mx[MT];
  bool raise = false;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    mx[i] = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx[i] = fmaxf(mx[i], s[i][kt][e]);
    raise = raise | (mx[i] * scale2 > m[i] + kSlack);
  }
  if (ballot(raise)) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      mx[i] = quad_max(mx[i]) * scale2;
      const float to = mx[i] > m[i] + kSlack ? mx[i] : m[i];
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

// Query operands of MT column tiles from column m0 of the job on; columns past its
// last and dimensions past D are zeros.
template <typename C, typename Tv, int MT, typename RowHead>
__device__ __forceinline__ void pa_queries(u32x4_t (&q)[MT][C::QR], const PaArgs& a, const PaJob& j,
                                           RowHead&& rowhead, int m0) {
  const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = m0 + 16 * i + r;
    const Tv* const qr = static_cast<const Tv*>(a.q) + (m < j.m_n ? rowhead(m) : 0) * a.D;
#pragma unroll
    for (int s = 0; s < C::QR; ++s) {
      const int d = (4 * s + q4) * C::VE;
      q[i][s] = u32x4_t{0, 0, 0, 0};
      if (m < j.m_n && d < a.D) q[i][s] = (*reinterpret_cast<const u32x4_t*>(qr + d) & a.keep) ^ a.flip;
    }
  }
}

// Four values of a row's result, D a multiple of 8 and the row on 16 bytes.
__device__ __forceinline__ void pa_put(uint16_t* dst, f32x4_t o) {
  const uint32_t lo = (uint32_t)f32_to_bf16(o[0]) | (uint32_t)f32_to_bf16(o[1]) << 16;
  const uint32_t hi = (uint32_t)f32_to_bf16(o[2]) | (uint32_t)f32_to_bf16(o[3]) << 16;
  *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
}
__device__ __forceinline__ void pa_put(float* dst, f32x4_t o) { *reinterpret_cast<f32x4_t*>(dst) = o; }
__device__ __forceinline__ float pa_lse(float m, float l) {
  return l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// WHOLE: the job is a row's whole work, and the block writes the result.
template <typename Tv, int DP, int MT, int W, bool WHOLE = false>
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
  if (!WHOLE && j.lo >= j.hi) {                  // no keys: this split adds nothing
    for (int m = threadIdx.x; m < j.m_n; m += (64 * W))
      a.part_ml[j.split * RH + rowhead(m)] = make_float2(-INFINITY, 0.f);
    return;
  }
  u32x4_t q[MT][C::QR];
  pa_queries<C, Tv>(q, a, j, rowhead, 0);
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
  // steps of the first range, then those of the second
  const int64_t first = j.hi > j.lo ? (j.hi - j.lo + C::KEYS - 1) / C::KEYS : 0;
  const int64_t steps = WHOLE ? first + (j.hi2 + C::KEYS - 1) / C::KEYS : first;
  auto load = [&](int64_t st) {
    const bool two = WHOLE && st >= first;
    const int64_t key = two ? (st - first) * C::KEYS : j.lo + st * C::KEYS;
    C::load(k, two ? j.k2 : j.k, key, two ? j.hi2 : j.hi, stride, a.D);
    C::load(v, two ? j.v2 : j.v, key, two ? j.hi2 : j.hi, stride, a.D);
  };
  if (wave < steps) load(wave);
  for (int64_t st = wave; st < steps; st += W) {
    f32x4_t s[MT][KT];
    C::template scores<MT>(s, q, k);
    C::stage(mine, v);
    if (st + W < steps) load(st + W);
    const int64_t left = WHOLE && st >= first ? j.hi2 - (st - first) * C::KEYS
                                              : j.hi - j.lo - st * C::KEYS;
    pa_softmax(s, m_run, l_run, o, a.scale2, (int)min(left, (int64_t)C::KEYS));
    lds_fence();
    C::template values<MT>(o, s, mine);
    lds_fence();
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
    for (int w = 1; w < W; ++w) top = fmaxf(top, s_m[w][m]);
    const float mu = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m_run[i] - mu);
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) l += s_l[w][m] * __builtin_amdgcn_exp2f(s_m[w][m] - mu);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) part[(wave * DT + dt) * kWave + lane] = o[i][dt] * f;
    __syncthreads();
    if (m < j.m_n) {
      const int64_t at = WHOLE ? rowhead(m) : j.split * RH + rowhead(m);
      if (wave == 0 && q4 == 0) {
        if (!WHOLE) a.part_ml[at] = make_float2(top, l);
        else if (a.lse) a.lse[at] = pa_lse(top, l);
      }
      for (int dt = wave; dt < DT; dt += W) {
        f32x4_t sum = part[dt * kWave + lane];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += part[(w * DT + dt) * kWave + lane];
        const int d = 16 * dt + 4 * q4;          // D is a multiple of 8
        if (d >= a.D) continue;
        if constexpr (WHOLE) pa_put(static_cast<Tv*>(a.out) + at * a.D + d, sum * (l == 0.f ? 0.f : 1.f / l));
        else *reinterpret_cast<f32x4_t*>(a.part_o + at * a.D + d) = sum;
      }
    }
    __syncthreads();                             // part is rewritten next
  }
}

// Many columns (a batch behind one prompt): every wave has MT column tiles of its
// own and goes over all keys of the block, which are staged in LDS for all of them,
// 32 keys at a time in two buffers; two more steps are in flight in registers. Keys
// are then loaded once for 16 * MT * W columns, and MFMAs bound the kernel with the
// exponentials beside them, where waves that split the keys would each wait for
// their own.
template <int DP, int MT, int W>
__device__ __forceinline__ void pa_rows_block(const PaArgs& a, const PaJob& j, char* lds) {
  using Tv = uint16_t;
  using C = PaCore<Tv, DP>;
  constexpr int KEYS = 32, CH = C::CHUNKS, DT = C::DT;
  constexpr int NL = (KEYS * CH + 64 * W - 1) / (64 * W);   // 16-byte chunks of K a thread, and of V
  constexpr int kTile = KEYS * DP * 2;
  const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t RH = a.R * a.Hq;
  auto rowhead = [&](int m) {
    return (j.row0 + (j.m0 + m) / a.nq) * a.Hq + j.h * a.nq + (j.m0 + m) % a.nq;
  };
  if (j.lo >= j.hi) {                            // no keys: this split adds nothing
    for (int m = threadIdx.x; m < j.m_n; m += (64 * W))
      a.part_ml[j.split * RH + rowhead(m)] = make_float2(-INFINITY, 0.f);
    return;
  }
  const int m0 = wave * 16 * MT;
  u32x4_t q[MT][C::QR];
  pa_queries<C, Tv>(q, a, j, rowhead, m0);
  f32x4_t o[MT][DT];
  float m_run[MT], l_run[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[i][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // K chunks XORed with the row, so that sixteen rows' reads of one chunk meet
  // different banks; V as PaCore::stage does
  auto swz_k = [](int row) { return DP == 64 ? (row >> 1) & 7 : row & 15; };
  const uint32_t stride = (uint32_t)(a.Hkv * a.D * 2);
  struct Regs { u32x4_t k[NL], v[NL]; };
  auto load = [&](Regs& x, int64_t key) {        // keys past hi: zeros
    const int64_t n = min(max(j.hi - key, (int64_t)1), (int64_t)KEYS);
    const int64_t from = min(key, j.hi - 1);
    const int bytes = (int)((uint32_t)(n - 1) * stride + (uint32_t)a.D * 2);
    const rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(j.k + from * stride), 0, bytes, 0x00027000);
    const rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(j.v + from * stride), 0, bytes, 0x00027000);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int at = threadIdx.x + i * (64 * W), row = at / CH, c = at % CH;
      const uint32_t off = c * 8 < a.D && row < KEYS ? (uint32_t)row * stride + c * 16 : kPastEnd;
      x.k[i] = buf_load16<false>(rk, off, 0);
      x.v[i] = buf_load16<false>(rv, off, 0);
    }
  };
  auto store = [&](const Regs& x, char* buf) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int at = threadIdx.x + i * (64 * W), row = at / CH, c = at % CH;
      if (KEYS * CH < 64 * W && row >= KEYS) break;
      *reinterpret_cast<u32x4_t*>(buf + (row * CH + (c ^ swz_k(row))) * 16) = x.k[i];
      *reinterpret_cast<u32x4_t*>(buf + kTile + (row * CH + (c ^ C::swz(row))) * 16) = x.v[i];
    }
  };
  auto barrier = []() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  auto step = [&](const char* buf, int64_t key) {
    f32x4_t s[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[i][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int t = 0; t < C::QR; ++t) {
        const int row = 16 * kt + r;
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(
            buf + (row * CH + ((4 * t + q4) ^ swz_k(row))) * 16);
#pragma unroll
        for (int i = 0; i < MT; ++i) C::mfma(s[i][kt], k, q[i][t]);
      }
    pa_softmax(s, m_run, l_run, o, a.scale2, (int)min(j.hi - key, (int64_t)KEYS));
    C::template values<MT>(o, s, buf + kTile);
  };
  char* const buf0 = lds;
  char* const buf1 = lds + 2 * kTile;
  Regs x0, x1;
  load(x0, j.lo);
  load(x1, j.lo + KEYS);
  store(x0, buf0);
  load(x0, j.lo + 2 * KEYS);
  barrier();
  for (int64_t key = j.lo;; key += 2 * KEYS) {
    store(x1, buf1);
    load(x1, key + 3 * KEYS);
    step(buf0, key);
    barrier();
    if (key + KEYS >= j.hi) break;
    store(x0, buf0);
    load(x0, key + 4 * KEYS);
    step(buf1, key + KEYS);
    barrier();
    if (key + 2 * KEYS >= j.hi) break;
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const float l = quad_sum(l_run[i]);
    const int m = m0 + 16 * i + r;
    if (m >= j.m_n) continue;
    const int64_t at = j.split * RH + rowhead(m);
    if (q4 == 0) a.part_ml[at] = make_float2(m_run[i], l);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int d = 16 * dt + 4 * q4;            // D is a multiple of 8
      if (d < a.D) *reinterpret_cast<f32x4_t*>(a.part_o + at * a.D + d) = o[i][dt];
    }
  }
}

// MT: 16-column tiles of a prefix block (ROWS: of each of its waves); suffix blocks
// have one. Two waves a SIMD hide each other's waits, so many columns go to eight
// waves of two tiles (four waves of four tiles, one a SIMD, whose accumulators also
// travel between the two halves of the register file: 64 rows of four heads behind
// 65536 keys 283 us).
constexpr int pa_waves(bool rows) { return rows ? 8 : 4; }
constexpr int pa_columns(int mt, bool rows) { return 16 * mt * (rows ? pa_waves(true) : 1); }
constexpr int pa_occupancy(int elt, int mt, int dp, bool rows) {
  return rows ? 2 : mt == 4 || dp == 256 ? 1 : mt == 1 && elt * dp <= 256 ? 3 : 2;
}

template <typename Tv, int DP, int MT, bool ROWS>
__global__ void __launch_bounds__(64 * pa_waves(ROWS), pa_occupancy(sizeof(Tv), MT, DP, ROWS))
pa_kernel(PaArgs a) {
  using C = PaCore<Tv, DP>;
  constexpr int W = pa_waves(ROWS);
  __shared__ __attribute__((aligned(16))) char lds[W * C::kStage];
  __shared__ float s_m[W][64], s_l[W][64];
  static_assert(C::kStage >= C::DT * kWave * 16, "O of the waves");
  static_assert(!ROWS || W * C::kStage >= 4 * 32 * DP * 2, "two buffers of K and V");
  PaJob j;
  if (!find_job<Tv, pa_columns(MT, ROWS)>(a, blockIdx.x, j)) return;
  if ((int64_t)blockIdx.x >= a.blocks_p) {
    pa_block<Tv, DP, 1, W>(a, j, lds, s_m, s_l);
  } else if constexpr (ROWS) {
    pa_rows_block<DP, MT, W>(a, j, lds);
  } else {
    pa_block<Tv, DP, MT, W>(a, j, lds, s_m, s_l);
  }
}

// A row and key head a block, prefix and suffix in one go, the result written: one
// launch where the keys are few.
constexpr int pa_row_waves(int dp) { return dp == 256 ? 4 : 8; }

template <typename Tv, int DP>
__global__ void __launch_bounds__(64 * pa_row_waves(DP))
pa_row_kernel(PaArgs a) {
  using C = PaCore<Tv, DP>;
  constexpr int W = pa_row_waves(DP);
  __shared__ __attribute__((aligned(16))) char lds[W * C::kStage];
  __shared__ float s_m[W][64], s_l[W][64];
  static_assert(C::kStage >= C::DT * kWave * 16, "O of the waves");
  PaJob j;
  if (!find_row<Tv>(a, blockIdx.x, j)) return;
  pa_block<Tv, DP, 1, W, true>(a, j, lds, s_m, s_l);
}

// Row r, head h: the splits' O, sums and maxima joined. tpr threads (at least
// D / 4) take four dimensions each, sg groups of them share the splits (both powers
// of two), so that a thread has few loads in a row: these launches are latency.
template <typename Tv>
__global__ void __launch_bounds__(kJoinThreads)
pa_join_kernel(PaArgs a, int tpr_shift, int sg_shift) {
  __shared__ f32x4_t s_o[kJoinThreads];
  __shared__ float2 s_ml[kJoinThreads];
  const int64_t RH = a.R * a.Hq;
  const int tpr = 1 << tpr_shift, sg = 1 << sg_shift;
  const int64_t at = (int64_t)blockIdx.x * (kJoinThreads >> (tpr_shift + sg_shift)) +
                     (threadIdx.x >> (tpr_shift + sg_shift));
  const int d = 4 * (threadIdx.x & (tpr - 1)), g = (threadIdx.x >> tpr_shift) & (sg - 1);
  const int64_t row = at / a.Hq;
  const bool live = at < RH && row >= group_row(a, 0) && row < group_row(a, a.G);
  const int n = a.splits_p + a.splits_s;
  float m = -INFINITY, l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  if (live && d < a.D) {
#pragma unroll 4
    for (int p = g; p < n; p += sg) {
      const float2 ml = a.part_ml[p * RH + at];
      const f32x4_t po = *reinterpret_cast<const f32x4_t*>(a.part_o + (p * RH + at) * a.D + d);
      if (ml.y == 0.f) continue;                 // a split without keys wrote no O
      const float top = fmaxf(m, ml.x), mu = top == -INFINITY ? 0.f : top;
      const float f0 = __builtin_amdgcn_exp2f(m - mu), f1 = __builtin_amdgcn_exp2f(ml.x - mu);
      l = l * f0 + ml.y * f1;
      o = o * f0 + po * f1;
      m = top;
    }
  }
  if (sg > 1) {
    s_o[threadIdx.x] = o;
    s_ml[threadIdx.x] = make_float2(m, l);
    __syncthreads();
    if (g != 0) return;
    for (int i = 1; i < sg; ++i) {               // in split group order
      const float2 ml = s_ml[threadIdx.x + (i << tpr_shift)];
      if (ml.y == 0.f) continue;
      const float top = fmaxf(m, ml.x), mu = top == -INFINITY ? 0.f : top;
      const float f0 = __builtin_amdgcn_exp2f(m - mu), f1 = __builtin_amdgcn_exp2f(ml.x - mu);
      l = l * f0 + ml.y * f1;
      o = o * f0 + s_o[threadIdx.x + (i << tpr_shift)] * f1;
      m = top;
    }
  }
  if (!live || d >= a.D) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  o *= inv;
  pa_put(static_cast<Tv*>(a.out) + at * a.D + d, o);
  if (a.lse && d == 0) a.lse[at] = pa_lse(m, l);
}

struct PaPlan {
  int mt, dp, splits_p, splits_s, tiles_s;
  int tpr_shift, sg_shift;                       // of the join
  bool rows, whole;                              // whole: a launch of rows, no splits
  int64_t slots_p, blocks_p, blocks_s;
  size_t o, ml, total;
};

int64_t pa_join_blocks(int64_t R, int64_t Hq, const PaPlan& pl) {
  return ceil_div(R * Hq, kJoinThreads >> (pl.tpr_shift + pl.sg_shift));
}

// Column tiles of a key-splitting block: the most that leaves every instance
// without a spilled register.
constexpr int pa_max_tiles(int elt, int dp) {
  return dp == 256 ? 1 : dp == 128 && elt == 4 ? 2 : 4;
}

PaPlan pa_plan(int64_t R, int64_t G, int32_t Hq, int32_t Hkv, int32_t D, int64_t P, int64_t S,
               int32_t dtype) {
  PaPlan pl{};
  const int nq = Hq / Hkv;
  pl.dp = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  const int64_t cols = ceil_div(R, G) * nq;      // of an average group
  pl.rows = dtype == MOE_BF16 && pl.dp <= 128 && cols > 64;
  if (pl.rows) pl.mt = cols <= 128 ? 1 : 2;
  else pl.mt = std::min(cols <= 16 ? 1 : cols <= 32 ? 2 : 4,
                        pa_max_tiles(dtype == MOE_BF16 ? 2 : 4, pl.dp));
  const int bm = pa_columns(pl.mt, pl.rows);
  pl.slots_p = R * nq / bm + G;
  pl.tiles_s = (int)ceil_div(nq, 16);
  auto splits = [](int64_t blocks, int64_t keys, int64_t want) {
    if (keys == 0) return 0;
    const int64_t most = std::min<int64_t>(ceil_div(keys, 128), 64);
    return (int)std::min(most, std::max<int64_t>(1, ceil_div(want, blocks)));
  };
  // the tiles of even groups (the upper bound counts one more a group); blocks of
  // many registers are one a compute unit, and a second round of them costs more
  // than the join of fewer splits saves
  const int64_t used = G * ceil_div(cols, bm);
  pl.splits_p = splits(used * Hkv, P, pl.rows && pl.mt == 2 ? 256 : 512);
  pl.splits_s = splits(R * Hkv * pl.tiles_s, S, 512);
  pl.blocks_p = ceil_div(pl.slots_p * pl.splits_p, 8) * 8 * Hkv;
  pl.blocks_s = ceil_div(R * pl.tiles_s * pl.splits_s, 8) * 8 * Hkv;
  pl.tpr_shift = pl.dp == 64 ? 4 : pl.dp == 128 ? 5 : 6;
  while (pl.sg_shift < 8 - pl.tpr_shift && (2 << pl.sg_shift) <= pl.splits_p + pl.splits_s)
    ++pl.sg_shift;
  // a step's loads take some 2.5 us, which two of a wave may cost against a launch and
  // the join; and while the blocks run at once, loads of a shared prefix by each of its
  // rows meet in the caches (4 rows behind 250 keys 9.4 us, split 6.8 + 4.2, behind 777
  // 16.6, 7.2 + 4.5; 64 rows of eight key heads 17.3, 16.3 + 4.1; 256 rows 63, 45 + 6.6).
  // At the limit the kernels are level (one or four rows behind 480 keys 12.0 and 12.4,
  // split 6.8 + 4.8 and 6.8 + 4.5), and the launch saved is the gain.
  const int64_t keys = dtype == MOE_BF16 ? 32 : 16;
  pl.whole = R * Hkv * pl.tiles_s <= 512 &&
             ceil_div(P, keys) + ceil_div(S, keys) <= 2 * pa_row_waves(pl.dp);
  // Splits change with the rows, and a call may need more of a workspace than a larger
  // one does. So `total` allows each cache as many rows of splits as any call of fewer
  // rows, groups or keys can have: with b blocks a split, ceil(want / b) splits of R rows
  // are at most R + (want - 1) R / b rows, and b is at least R Hkv tiles_s of suffixes,
  // R Hq / bm of prefixes.
  auto rows = [&](int64_t keys, int64_t more) {
    return keys == 0 ? 0 : std::min(R * std::min<int64_t>(ceil_div(keys, 128), 64), R + more);
  };
  const bool any_rows = dtype == MOE_BF16 && pl.dp <= 128;
  const int64_t want_bm =                        // the most of any column class
      any_rows ? 512 * pa_columns(1, true)
               : 512 * pa_columns(pa_max_tiles(dtype == MOE_BF16 ? 2 : 4, pl.dp), false);
  const size_t n = (size_t)(rows(P, want_bm / Hq) + rows(S, 512 / (Hkv * pl.tiles_s))) * Hq;
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
  // a launch's dimension is below 2^32 threads
  return pl.whole || (pl.blocks_p + pl.blocks_s < 2 * lim / (64 * pa_waves(pl.rows)) &&
                      pa_join_blocks(R, Hq, pl) < 2 * lim / kJoinThreads);
}

template <typename Tv, int DP>
int pa_launch(const PaArgs& a, const PaPlan& pl, unsigned blocks, hipStream_t st) {
  constexpr int M = pa_max_tiles(sizeof(Tv), DP);
  if constexpr (sizeof(Tv) == 2 && DP <= 128) {
    if (pl.rows) {
      constexpr int T = 64 * pa_waves(true);
      if (pl.mt == 1) pa_kernel<Tv, DP, 1, true><<<dim3(blocks), dim3(T), 0, st>>>(a);
      else pa_kernel<Tv, DP, 2, true><<<dim3(blocks), dim3(T), 0, st>>>(a);
      MOE_CHECK_LAUNCH();
      return MOE_OK;
    }
  }
  constexpr int T = 64 * pa_waves(false);
  if (pl.mt == 1) pa_kernel<Tv, DP, 1, false><<<dim3(blocks), dim3(T), 0, st>>>(a);
  if constexpr (M >= 2)
    if (pl.mt == 2) pa_kernel<Tv, DP, 2, false><<<dim3(blocks), dim3(T), 0, st>>>(a);
  if constexpr (M >= 4)
    if (pl.mt == 4) pa_kernel<Tv, DP, 4, false><<<dim3(blocks), dim3(T), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv>
int pa_run(const PaArgs& a, const PaPlan& pl, hipStream_t st) {
  if (pl.whole) {
    const dim3 grid((unsigned)(a.R * a.Hkv * a.tiles_s));
    if (pl.dp == 64) pa_row_kernel<Tv, 64><<<grid, dim3(64 * pa_row_waves(64)), 0, st>>>(a);
    else if (pl.dp == 128) pa_row_kernel<Tv, 128><<<grid, dim3(64 * pa_row_waves(128)), 0, st>>>(a);
    else pa_row_kernel<Tv, 256><<<grid, dim3(64 * pa_row_waves(256)), 0, st>>>(a);
    MOE_CHECK_LAUNCH();
    return MOE_OK;
  }
  const unsigned blocks = (unsigned)(pl.blocks_p + pl.blocks_s);
  int rc = MOE_OK;
  if (blocks) {
    rc = pl.dp == 64 ? pa_launch<Tv, 64>(a, pl, blocks, st)
       : pl.dp == 128 ? pa_launch<Tv, 128>(a, pl, blocks, st)
                      : pa_launch<Tv, 256>(a, pl, blocks, st);
  }
  if (rc != MOE_OK) return rc;
  pa_join_kernel<Tv><<<dim3((unsigned)pa_join_blocks(a.R, a.Hq, pl)), dim3(kJoinThreads), 0, st>>>(
      a, pl.tpr_shift, pl.sg_shift);
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
  MOE_CHECK_ARG(isfinite(scale * kLog2e));       // scores are held times log2 e
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
  // never 0, which would make a masked key's score NaN: then the queries are zeros
  const bool none = fabsf(scale) < 1e-37f;
  a.scale2 = none ? 1.f : fabsf(scale) * kLog2e;
  a.keep = none ? 0u : ~0u;
  a.flip = none || scale >= 0.f ? 0u : dtype == MOE_BF16 ? 0x80008000u : 0x80000000u;
  a.splits_p = pl.splits_p;
  a.splits_s = pl.splits_s;
  a.blocks_p = pl.blocks_p;
  a.slots_p = pl.slots_p;
  a.tiles_s = pl.tiles_s;
  a.part_o = reinterpret_cast<float*>(ws + pl.o);
  a.part_ml = reinterpret_cast<float2*>(ws + pl.ml);
  a.out = out;
  a.lse = lse;
  hipStream_t st = as_stream(stream);
  return dtype == MOE_BF16 ? pa_run<uint16_t>(a, pl, st) : pa_run<float>(a, pl, st);
}
