// moe_prompt_attention: causal attention of packed sequences.
//
// Bound by the matrix cores where prompts are long: 4 D Hq flop a visible pair of
// tokens, against K and V read once. The queries of a sequence that read one key head
// (tokens x query heads of it, so that the tokens a tile spans and with them what the
// diagonal wastes are few) are the columns of the products:
//   S^T = K Q^T     rows: keys, columns: queries
//   O^T = V^T P^T   rows: values' dimensions, columns: queries
// Transposed so, a lane of the MFMA result holds scores of one query for four
// neighbouring keys: the running maximum and sum are one register each, the
// rescaling of O is lane by lane, and the scores of two 16-key tiles are, in
// place, a lane's eight operands of the second product (its k slots 8q + j are
// keys 4q + j of the first tile and 4q + j - 4 of the second). V^T comes from LDS
// through the transposing read, four keys of one column at a time.
// Every wave has 16 or 32 columns of its own; keys and values go straight from memory to
// LDS, a tile of keys ahead of the one that all waves of a block compute on, swizzled by
// which 16 bytes each lane fetches. Tiles before the first query of a wave need no
// mask. One prompt of 16384 tokens, 32 heads of 128 over eight key heads, takes 1.86 ms
// (1.93 on another card): 1183 TFLOP/s, the MFMAs run in 51 % of the cycles,
// instructions are issued in 71 %. Times here and below are of calls in a captured graph.
// Measured and left out: another order of MFMAs and exponentials (the tiles of columns
// apart, interleaved by hand), reads from LDS further ahead, a third buffer, priorities
// between the waves of a SIMD: level or slower.
#include "moeflow_prompt.h"
#include "attention.h"
#include "dma.h"
#include "spans.h"

#include <algorithm>
#include <type_traits>

namespace moe {
namespace {

constexpr uint32_t kPastEnd = 0xfffffff0u;       // no buffer here is as long
constexpr int kLook = 2;                         // of s_odd: values are to be looked at again

struct PrArgs {
  const void *q, *k, *v;
  const int32_t *q_offsets, *k_offsets;
  int64_t N, M, B, q_stride, k_stride, v_stride; // strides in elements
  int Hq, Hkv, D, nq;                            // nq: query heads of a key head
  float per_nq;                                  // 1 / nq
  float scale2;                                  // |scale| log2 e
  uint32_t keep, flip;
  int splits;
  int64_t slots;                                 // row tiles (upper bound)
  float* part_o;                                 // [splits][N * Hq][D]
  float2* part_ml;                               // [splits][N * Hq]
  void* out;
  float* lse;
};

__device__ __forceinline__ int64_t pr_offset(const int32_t* o, int64_t b, int64_t n) {
  if (!o) return b == 0 ? 0 : n;
  return min(max((int64_t)o[b], (int64_t)0), n);
}

// What a block works on: columns m0 .. m0 + m_n - 1 (column m is token m / nq of the
// sequence, query head h * nq + m % nq), keys [lo, hi) of the sequence.
struct PrJob {
  const char *k, *v;                             // of key 0, head h
  int64_t row0;                                  // the sequence's first row of q
  int lo, hi, past, m0, cols;                    // past: keys before the first query's own
  int tok0, rem0;                                // token and query head of column m0
  int h, split;
};

// Token of column m0 + off, off below 2^16: (x + 1/2) / nq lies 1 / (2 nq) or more from
// a whole number, float32 is off by less.
__device__ __forceinline__ int pr_token(const PrArgs& a, const PrJob& j, int off) {
  return j.tok0 + (int)(((float)(j.rem0 + off) + 0.5f) * a.per_nq);
}

// Row tiles of sequence b start at slot floor(first row * nq / BM) + b: slots of
// different sequences never meet, and a wave finds a slot's sequence in steps of 64
// probes. Later tiles, which see more keys, come first; head h goes to XCD h % 8, so
// that the tiles of a head share its keys in one L2.
template <typename Tv, int BM, int BN>
__device__ __forceinline__ bool pr_find(const PrArgs& a, PrJob& j) {
  uint32_t u = blockIdx.x / (uint32_t)a.Hkv;
  j.h = (int)(blockIdx.x - u * (uint32_t)a.Hkv);
  j.split = 0;
  if (a.splits > 1) {
    j.split = (int)(u % (uint32_t)a.splits);
    u /= (uint32_t)a.splits;
  }
  const int64_t slot = a.slots - 1 - u;
  int64_t b = 0, n = a.B;
  const int lane = lane_id();
  while (n > 1) {
    const int64_t step = (n + 63) / 64, at = b + lane * step;
    const bool in = at < b + n && pr_offset(a.q_offsets, at, a.N) * a.nq / BM + at <= slot;
    const int c = max((int)__popcll(ballot(in)) - 1, 0);
    b += c * step;
    n = min(step, n - c * step);
  }
  const int64_t r0 = pr_offset(a.q_offsets, b, a.N), r1 = pr_offset(a.q_offsets, b + 1, a.N);
  const int64_t k0 = pr_offset(a.k_offsets, b, a.M);
  const int64_t keys = max(pr_offset(a.k_offsets, b + 1, a.M) - k0, (int64_t)0);
  const int64_t tile = slot - (r0 * a.nq / BM + b);
  j.cols = (int)((r1 - r0) * a.nq);              // N * Hq < 2^31
  if (tile < 0 || tile * BM >= j.cols) return false;
  j.m0 = (int)tile * BM;
  j.row0 = r0;
  j.past = (int)(keys - (r1 - r0));
  j.tok0 = (int)((uint32_t)j.m0 / (uint32_t)a.nq);
  j.rem0 = j.m0 - j.tok0 * a.nq;
  const int end = max(j.past + pr_token(a, j, min(BM, j.cols - j.m0) - 1) + 1, 0);
  j.lo = 0;
  j.hi = end;
  if (a.splits > 1) {
    const uint32_t per = (((uint32_t)end + a.splits - 1) / (uint32_t)a.splits + BN - 1) / BN * BN;
    j.lo = (int)min((uint64_t)end, (uint64_t)per * j.split);
    j.hi = (int)min((uint32_t)end, j.lo + per);
  }
  j.k = reinterpret_cast<const char*>(static_cast<const Tv*>(a.k) + k0 * a.k_stride +
                                      (int64_t)j.h * a.D);
  j.v = reinterpret_cast<const char*>(static_cast<const Tv*>(a.v) + k0 * a.v_stride +
                                      (int64_t)j.h * a.D);
  return true;
}

// DP: the dimension padded to rows of whole 128 bytes; 16-byte chunks past D are zeros.
template <typename Tv, int DP, int kMT, int W, int BN>
struct PrCore {
  static constexpr bool BF16 = sizeof(Tv) == 2;
  static constexpr int VE = 16 / sizeof(Tv);     // values per chunk
  static constexpr int CH = DP / VE;             // chunks of a row
  static constexpr int QR = CH / 4;              // operands of a query: chunk 4t + q4
  static constexpr int DT = DP / 16, KT = BN / 16;
  static constexpr int kTile = BN * CH * 16;     // bytes of a tile of keys, or of values
  static constexpr int PIECES = kTile / 1024 / W;   // 1 KB pieces a wave loads of a tile
  static_assert(kTile % (1024 * W) == 0, "whole pieces");

  // Chunk c of row r lies at c ^ swz: sixteen rows' reads of one chunk (keys), and
  // the transposing reads' eight rows x 32 bytes (values), meet different banks.
  static __device__ __forceinline__ int swz_k(int row) { return CH == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int swz_v(int row) {
    if constexpr (!BF16) return 4 * ((row >> 2) & 3);
    return CH == 8 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
  }
  // Byte offsets of the chunks that a lane loads, from a tile's first key on.
  static __device__ __forceinline__ void offsets(uint32_t (&k)[PIECES], uint32_t (&v)[PIECES],
                                                 int wave, const PrArgs& a) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int g = (wave * PIECES + p) * 64 + lane_id(), row = g / CH, c = g % CH;
      const int ck = c ^ swz_k(row), cv = c ^ swz_v(row);
      k[p] = ck * VE < a.D ? (uint32_t)row * (uint32_t)(a.k_stride * sizeof(Tv)) + ck * 16 : kPastEnd;
      v[p] = cv * VE < a.D ? (uint32_t)row * (uint32_t)(a.v_stride * sizeof(Tv)) + cv * 16 : kPastEnd;
    }
  }
  // Keys from `key` on into LDS, those from `end` on as zeros.
  static __device__ __forceinline__ void load(uint32_t lds, const char* base, int64_t stride, int key,
                                              int end, int D, const uint32_t (&off)[PIECES],
                                              int wave) {
    const u32x4_t rs = dma_rows(base, key, min(end - key, BN), (uint32_t)(stride * (int64_t)sizeof(Tv)),
                                (uint32_t)D * sizeof(Tv));
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
      dma<16>(lds + (wave * PIECES + p) * 1024, off[p], rs);
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
  static __device__ __forceinline__ void scores(f32x4_t (&s)[kMT][KT], const u32x4_t (&q)[kMT][QR],
                                                const char* lds) {
    const int r = lane_id() & 15, q4 = lane_id() >> 4;
    const int at = r * CH + (q4 ^ swz_k(r));     // rows 16 apart share swz
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < kMT; ++i) s[i][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < QR; ++t) {
      const char* const from = lds + (at ^ (4 * t)) * 16;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(from + kt * 16 * CH * 16);
#pragma unroll
        for (int i = 0; i < kMT; ++i) mfma(s[i][kt], k, q[i][t]);
      }
    }
  }
  // p, rounded to bf16 (by at most 2^-8 of it, for the matrix cores); its sum is taken of
  // the float32 values. Of flat attention over 1000 or 8192 keys the result is off by
  // 2.3e-3 (rms), 1.7e-3 of it the rounding of the result itself. With p as the sum of two
  // bf16 numbers only that is left, and 777 tokens take 23.9 us for 20.3, sixteen prompts
  // of up to 1000 144 for 126, one of 16384 2.73 ms for 1.93.
  static __device__ __forceinline__ u32x4_t numerators(const f32x4_t& p0, const f32x4_t& p1) {
    bf16x8_t b;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      b[e] = (__bf16)p0[e];
      b[e + 4] = (__bf16)p1[e];
    }
    return __builtin_bit_cast(u32x4_t, b);
  }
  // O += V^T P^T
  static __device__ __forceinline__ void values(f32x4_t (&o)[kMT][DT], const f32x4_t (&p)[kMT][KT],
                                                const char* lds) {
    const int r = lane_id() & 15, q4 = lane_id() >> 4;
    if constexpr (BF16) {
      u32x4_t pb[kMT][KT / 2];
#pragma unroll
      for (int i = 0; i < kMT; ++i)
#pragma unroll
        for (int g = 0; g < KT / 2; ++g) pb[i][g] = numerators(p[i][2 * g], p[i][2 * g + 1]);
      const int row = 4 * q4 + (r >> 2), at = row * CH + (((r >> 1) & 1) ^ swz_v(row));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const char* const from = lds + (at ^ (2 * dt)) * 16 + (r & 1) * 8;
#pragma unroll
        for (int g = 0; g < KT / 2; ++g) {
          s16x4_t v[2];
#pragma unroll
          for (int t = 0; t < 2; ++t)
            v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4_t*)(from + (2 * g + t) * 16 * CH * 16));
          const u32x4_t vt = __builtin_bit_cast(
              u32x4_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int i = 0; i < kMT; ++i) mfma(o[i][dt], vt, pb[i][g]);
        }
      }
    } else {
      const int row = 4 * q4, at = row * CH + ((r >> 2) ^ swz_v(row));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const char* const from = lds + (at ^ (4 * dt)) * 16 + (r & 3) * 4;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = *reinterpret_cast<const float*>(from + (16 * kt + e) * CH * 16);
#pragma unroll
            for (int i = 0; i < kMT; ++i)
              o[i][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[i][kt][e], o[i][dt], 0, 0, 0);
          }
      }
    }
  }
  // For every dimension the first key whose value is +inf or NaN, and -inf or NaN: a query
  // that sees it gets the infinity, or both, whatever the key's weight. Of eight (four)
  // values from dimension d0 on, which become 0 in x if it is to hold no others.
  static __device__ __forceinline__ bool is_odd(const u32x4_t& w) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      odd |= (w[e] & 0x7f800000u) == 0x7f800000u;
      if constexpr (BF16) odd |= (w[e] & 0x7f80u) == 0x7f80u;
    }
    return odd;
  }
  template <bool CLEAR, typename T>
  static __device__ __forceinline__ void note_odd(T* x, int d0, int key, int* up, int* down) {
#pragma unroll 1
    for (int e = 0; e < VE; ++e) {
      float f;
      if constexpr (BF16) f = bf16_to_f32(x[e]);
      else f = x[e];
      if (fabsf(f) < INFINITY) continue;
      if (!(f < 0.f)) atomicMin(up + d0 + e, key);
      if (!(f > 0.f)) atomicMin(down + d0 + e, key);
      if constexpr (CLEAR) x[e] = 0;
    }
  }
  // In a tile that some query does not see as a whole 0 times them would be NaN: those in
  // the chunks that this wave loaded become 0. *any: there are such (the end of a block
  // without them is 1 us shorter: 8 tokens 6.2 -> 5.2).
  static __device__ __forceinline__ void take_odd(char* tile, int key, int wave, int* up, int* down,
                                                  int* any) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int g = (wave * PIECES + p) * 64 + lane_id(), row = g / CH;
      u32x4_t* const at = reinterpret_cast<u32x4_t*>(tile) + g;
      if (!is_odd(*at)) continue;
      *any = 1;
      note_odd<true>(reinterpret_cast<Tv*>(at), ((g % CH) ^ swz_v(row)) * VE, key + row, up, down);
    }
  }
  // Other tiles are not looked at (one prompt of 16384 tokens 1.91 -> 2.07 ms, of 224 8.4
  // -> 9.8 us): theirs make O infinite or NaN, and then the block's threads look at the
  // values of all its keys once more. To see that costs 0.1 us of a call; a NaN among the
  // values of 16384 tokens then costs a fifth of it.
  static __device__ __forceinline__ bool finite(const f32x4_t (&o)[kMT][DT]) {
    float top[2] = {0.f, 0.f};                   // maxima that keep a NaN, two values each time
#pragma unroll
    for (int i = 0; i < kMT; ++i)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          top[dt % 2] = __builtin_elementwise_maximum(top[dt % 2], fabsf(o[i][dt][e]));
    return __builtin_elementwise_maximum(top[0], top[1]) < INFINITY;
  }
  static __device__ __forceinline__ void find_odd(const char* v, int64_t stride, int D, int lo, int hi,
                                                  int threads, int* up, int* down) {
    const int d0 = (int)threadIdx.x % CH * VE;
    if (d0 >= D) return;
#pragma unroll 1
    for (int key = lo + (int)threadIdx.x / CH; key < hi; key += threads / CH) {
      const Tv* const from = reinterpret_cast<const Tv*>(v) + key * stride + d0;
      if (is_odd(*reinterpret_cast<const u32x4_t*>(from))) note_odd<false>(from, d0, key, up, down);
    }
  }
};

// Keys of a tile: of 64 in blocks of four waves fewer blocks fit a compute unit (sixteen
// prompts of up to 1000 tokens 126 us, of 64 keys 154).
constexpr int pr_keys(int elt, int dp, int waves) {
  return elt * dp < 256 || (elt * dp == 256 && waves == 8) ? 64 : elt * dp <= 512 ? 32 : 16;
}

// KS groups of W waves have the same columns and take tiles of keys in turn; they are
// added up through LDS at the end.
template <typename Tv, int DP, int kMT, int W, int KS>
__global__ void __launch_bounds__(64 * W * KS, 2) pr_kernel(PrArgs a) {
  constexpr int BM = 16 * kMT * W, BN = pr_keys(sizeof(Tv), DP, W);
  using C = PrCore<Tv, DP, kMT, W, BN>;
  constexpr int KT = C::KT, DT = C::DT, QR = C::QR;
  constexpr int kPart = W * kMT * DT * kWave * 16;   // O of a group
  constexpr int kLds = KS > 1 && KS * kPart > 4 * KS * C::kTile ? KS * kPart : 4 * KS * C::kTile;
  __shared__ __attribute__((aligned(16))) char lds[kLds];
  __shared__ float s_m[KS][W * kMT * 16], s_l[KS][W * kMT * 16];
  __shared__ int s_up[DP], s_down[DP], s_odd;
  PrJob j;
  if (!pr_find<Tv, BM, BN>(a, j)) return;
  const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
  const int any = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wave = any % W, group = any / W;
  for (int d = threadIdx.x; d < DP; d += 64 * W * KS) s_up[d] = s_down[d] = 0x7fffffff;
  if (threadIdx.x == 0) s_odd = 0;
  uint32_t off_k[C::PIECES], off_v[C::PIECES];
  C::offsets(off_k, off_v, wave, a);
  char* const ring = lds + group * 4 * C::kTile;
  const uint32_t ring_at = lds_address(ring);
  auto load = [&](int buf, int key) {
    const uint32_t to = ring_at + buf * 2 * C::kTile;
    C::load(to, j.k, a.k_stride, key, j.hi, a.D, off_k, wave);
    C::load(to + C::kTile, j.v, a.v_stride, key, j.hi, a.D, off_v, wave);
  };
  const int key0 = j.lo + group * BN;            // the group's first tile
  if (key0 < j.hi) load(0, key0);
  const int w_off = wave * 16 * kMT, w_m = j.m0 + w_off;   // the wave's first column
  int last[kMT];                                 // of a column: its last key
  int64_t at[kMT];                               // its row and head
  u32x4_t q[kMT][QR];
#pragma unroll
  for (int i = 0; i < kMT; ++i) {
    const int off = w_off + 16 * i + r, tok = pr_token(a, j, off);
    const bool in = j.m0 + off < j.cols;
    const int head = j.h * a.nq + j.m0 + off - tok * a.nq;
    last[i] = in ? j.past + tok : -1;
    at[i] = (j.row0 + tok) * a.Hq + head;
    const Tv* const row = static_cast<const Tv*>(a.q) +
                          (in ? (j.row0 + tok) * a.q_stride + (int64_t)head * a.D : 0);
#pragma unroll
    for (int t = 0; t < QR; ++t) {
      const int d = (4 * t + q4) * C::VE;
      q[i][t] = u32x4_t{0, 0, 0, 0};
      if (in && d < a.D) q[i][t] = (*reinterpret_cast<const u32x4_t*>(row + d) & a.keep) ^ a.flip;
    }
  }
  // keys of the wave: none from w_hi on, all visible to all of its columns before w_all
  const int w_end = min(w_m + 16 * kMT, j.cols);
  const int w_hi = w_m < j.cols ? min(j.hi, j.past + pr_token(a, j, w_end - 1 - j.m0) + 1) : 0;
  const int w_all = w_end - w_m == 16 * kMT ? j.past + pr_token(a, j, w_off) + 1 : 0;
  // before which key no column of the block needs a mask
  const int b_all = j.m0 + BM <= j.cols ? j.past + j.tok0 + 1 : 0;

  f32x4_t o[kMT][DT];
  float m_run[kMT], l_run[kMT];
#pragma unroll
  for (int i = 0; i < kMT; ++i) {
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[i][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();
  // one tile of keys, in buffer BUF: known to the compiler, so that every LDS read is a
  // lane's address and a constant
  auto tile = [&](auto BUF, int key) {
    char* const tk = ring + BUF * 2 * C::kTile;
    wait_loads<0>();
    if (key < j.hi && key + BN > b_all) C::take_odd(tk + C::kTile, key, wave, s_up, s_down, &s_odd);
    // the tile has landed, and every wave is done with the other buffer
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (key + KS * BN < j.hi) load(1 - BUF, key + KS * BN);
    if (key >= w_hi) return;
    f32x4_t s[kMT][KT];
    C::scores(s, q, tk);
    if (key + BN > w_all) {
#pragma unroll
      for (int i = 0; i < kMT; ++i)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key + 16 * kt + 4 * q4 + e > last[i]) s[i][kt][e] = -INFINITY;
    }
    softmax_step<Tv>(s, m_run, l_run, o, a.scale2);
    C::values(o, s, tk + C::kTile);
  };
  // as many turns for every group: they meet at the barriers
  for (int key = j.lo; key < j.hi; key += 2 * KS * BN) {
    tile(std::integral_constant<int, 0>{}, key + group * BN);
    if (key + KS * BN < j.hi) tile(std::integral_constant<int, 1>{}, key + (KS + group) * BN);
  }
  float l_all[kMT];
#pragma unroll
  for (int i = 0; i < kMT; ++i) l_all[i] = quad_sum(l_run[i]);
  // take_odd is done: every wave has passed the last tile's barrier
  if (j.lo + BN <= b_all && !C::finite(o)) atomicOr(&s_odd, kLook);
  bool odd;
  auto look = [&]() {                            // after a barrier
    const int what = __builtin_amdgcn_readfirstlane(s_odd);
    odd = what != 0;
    if (!(what & kLook)) return;
    C::find_odd(j.v, a.v_stride, a.D, j.lo, j.hi, 64 * W * KS, s_up, s_down);
    __syncthreads();
  };
  if constexpr (KS > 1) {
#pragma unroll
    for (int i = 0; i < kMT; ++i)
      if (q4 == 0) {
        s_m[group][w_off + 16 * i + r] = m_run[i];
        s_l[group][w_off + 16 * i + r] = l_all[i];
      }
    __syncthreads();                             // and every wave is done with its tiles
    look();
    f32x4_t* const part = reinterpret_cast<f32x4_t*>(lds);
#pragma unroll
    for (int i = 0; i < kMT; ++i) {
      const int c = w_off + 16 * i + r;
      float top = s_m[0][c];
#pragma unroll
      for (int g = 1; g < KS; ++g) top = fmaxf(top, s_m[g][c]);
      const float mu = top == -INFINITY ? 0.f : top;
      const float f = __builtin_amdgcn_exp2f(m_run[i] - mu);
      l_all[i] = 0.f;
#pragma unroll
      for (int g = 0; g < KS; ++g) l_all[i] += s_l[g][c] * __builtin_amdgcn_exp2f(s_m[g][c] - mu);
      m_run[i] = top;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        o[i][dt] *= f;
        if (group > 0) part[((any * kMT + i) * DT + dt) * kWave + lane] = o[i][dt];
      }
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll 1
    for (int g = 1; g < KS; ++g)
#pragma unroll
      for (int i = 0; i < kMT; ++i)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          o[i][dt] += part[(((any + g * W) * kMT + i) * DT + dt) * kWave + lane];
  } else {
    __syncthreads();
    look();
  }
  const int64_t RH = a.N * a.Hq;
#pragma unroll
  for (int i = 0; i < kMT; ++i) {
    const float l = l_all[i];
    if (w_m + 16 * i + r >= j.cols) continue;
    const int64_t to = j.split * RH + at[i];
    const float f = a.splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
    // a split of no weight may hold infinities: its sum, of a maximum of -inf, adds 0
    if (q4 == 0) {
      if (a.splits > 1) a.part_ml[to] = make_float2(m_run[i], odd && l == 0.f ? 1.f : l);
      else if (a.lse) a.lse[to] = lse_of(m_run[i], l);
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int d = 16 * dt + 4 * q4;            // D is a multiple of 8
      if (d >= a.D) continue;
      f32x4_t x = {0.f, 0.f, 0.f, 0.f};          // of no weight, whatever the values hold
      if (l != 0.f) x = o[i][dt] * f;
      if (odd && (l != 0.f || a.splits > 1)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool up = last[i] >= s_up[d + e], down = last[i] >= s_down[d + e];
          // NaN of both, and of a sum that is NaN
          if (up || down) x[e] = (up ? INFINITY : 0.f) + (down ? -INFINITY : 0.f) + (l - l);
        }
      }
      if (a.splits > 1) *reinterpret_cast<f32x4_t*>(a.part_o + to * a.D + d) = x;
      else put4(static_cast<Tv*>(a.out) + to * a.D + d, x);
    }
  }
}

struct PrPlan {
  int dp, mt, waves, groups, splits;             // groups: of waves over one block's keys
  int64_t slots, blocks;
  size_t ml, total;
};

// Blocks of eight waves with 32 columns each load keys half as often and have the higher
// rate (one prompt of 16384 tokens, 32 heads of 128: 1.86 ms, of four waves with 16
// columns 2.17; 4096 tokens 136 and 155), but for few or short prompts smaller blocks
// fill the card better and cost less to start (777 tokens 20.1 us, wide 31.9; 2048 49 and
// 64; sixteen prompts of up to 1000 126 and 137, of up to 2000 level; 16 tokens 5.5 and
// 7.8).
constexpr int kWideKeys = 4096, kWideColumns = 256;
// Keys are split over blocks while at most this many blocks are then in flight (bf16,
// 64 tokens each of four sequences behind 4000 keys 34 us, with half as many 38; 777
// tokens in one group, whose 392 blocks are left whole, 24.6, in two splits 28.9: joins pay
// for keys that few queries see), each of kMinKeys at least (one token behind 2000 keys
// 11.4 us, of twice as many 13.3). float32 blocks take so long that more of them pay (two
// prompts of 1000 tokens, 8 heads of 128: three splits 60 us, two 84).
constexpr int kSplitBlocks = 512, kWideSplitBlocks = 256, kFloatSplitBlocks = 768;
constexpr int kMinKeys = 128, kMostSplits = 64;
// Two groups of waves on a block's columns while blocks do not fill the card and have
// enough keys (777 tokens 24.6 -> 20.1 us, 2000 of 16 heads of 256 93 -> 69, of 28 heads of
// 80 56 -> 42; 2048 tokens of 32 heads, 1024 blocks, 49 -> 58, 16 tokens 5.5 -> 6.5);
// float32 of more than 64 dimensions has no LDS for it (64 -> 74).
constexpr int kGroupBlocks = 896, kGroupKeys = 512;
// Four groups where every block has a compute unit to itself, which its LDS takes (32
// heads of 128: 256 tokens 14.9 -> 10.6 us, 400 19.0 -> 12.1, 512 20.2 -> 13.6; 128 tokens
// of 16 heads 6.9 -> 9.3; 600, in 304 blocks, 15.6 -> 18.6), and sequences have columns to
// fill it (16 tokens of two sequences behind 1000 keys 14.2 -> 16.8). A join then costs as
// much as four tiles a group: splits are of kFourMinKeys at least (512 tokens of 16 heads
// 12.8 us, in two splits 18.7; of 1024 keys, 40 tokens behind 3000 take 27.1 instead of
// 19.9). float32, whose splits are more, 31.9 -> 38.5 (1500 tokens of 4 heads of 64).
constexpr int kFourBlocks = 256, kFourKeys = 256, kFourColumns = 128, kFourMinKeys = 512;

PrPlan pr_plan(int64_t N, int64_t M, int64_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype) {
  PrPlan pl{};
  const int nq = Hq / Hkv;
  const int64_t keys = ceil_div(M, B);           // of an average sequence
  const bool wide = dtype == MOE_BF16 && keys >= kWideKeys && ceil_div(N, B) * nq >= kWideColumns;
  pl.dp = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  pl.waves = wide ? 8 : 4;
  pl.mt = wide && pl.dp < 256 ? 2 : 1;
  const int64_t bm = 16 * pl.mt * pl.waves;
  pl.slots = N * nq / bm + B;
  auto most = [](int64_t keys) {
    return std::min<int64_t>(std::max<int64_t>(1, keys / kMinKeys), kMostSplits);
  };
  // blocks of a split, if sequences are alike; those without a token have none
  const int64_t some = std::min(B, N), cols = ceil_div(N, some) * nq;
  const int64_t used = some * ceil_div(cols, bm) * Hkv;
  pl.groups = !wide && used <= kGroupBlocks && keys >= kGroupKeys &&
                      (dtype == MOE_BF16 || pl.dp == 64) ? 2 : 1;
  if (!wide && dtype == MOE_BF16 && pl.dp <= 128 && used <= kFourBlocks && keys >= kFourKeys &&
      cols >= kFourColumns)
    pl.groups = 4;
  const int64_t want = pl.groups == 4 ? kFourBlocks : wide ? kWideSplitBlocks
                     : dtype == MOE_F32 ? kFloatSplitBlocks : kSplitBlocks;
  const int64_t fit = pl.groups == 4 ? std::max<int64_t>(1, keys / kFourMinKeys) : most(keys);
  pl.splits = (int)std::min(std::min(fit, most(keys)), std::max<int64_t>(1, want / used));
  // a launch's threads are below 2^32; the slots are more than the tiles where sequences
  // are empty
  if (pl.slots * Hkv * pl.splits >= ((int64_t)1 << 32) / 1024) pl.splits = 1;
  pl.blocks = pl.slots * Hkv * pl.splits;
  // Splits of all rows are at most as many rows as the blocks have columns: `total` allows
  // every call for that many, and never falls as a call grows.
  constexpr int64_t kRows = std::max(std::max(kSplitBlocks, kFloatSplitBlocks) * 64,
                                     kWideSplitBlocks * 256);
  const int64_t rows = most(M) == 1 ? 0 : std::min(N * Hq * most(M), kRows);
  pl.ml = align_up((size_t)rows * D * 4, 256);
  pl.total = align_up(pl.ml + (size_t)rows * 8, 256);
  return pl;
}

bool pr_ok(int64_t N, int64_t M, int64_t B, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype) {
  return N >= 1 && M >= 0 && B >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && D >= 1 &&
         valid_dtype(dtype);
}
bool pr_supported(int64_t N, int64_t M, int64_t B, int32_t Hq, int32_t Hkv, int32_t D) {
  const int64_t lim = (int64_t)1 << 31;
  return D % 8 == 0 && D <= 256 && N < lim / Hq && M <= lim / 2 && B < lim &&
         (int64_t)Hq * D <= (1 << 24) && Hq <= (1 << 16) && N * Hq / 32 + (double)B * Hkv < (1 << 22);
}

template <typename Tv, int DP>
int pr_launch(const PrArgs& a, const PrPlan& pl, hipStream_t st) {
  const dim3 grid((unsigned)pl.blocks), block((unsigned)(64 * pl.waves * pl.groups));
  if constexpr (sizeof(Tv) == 2)
    if (pl.waves == 8) pr_kernel<Tv, DP, DP == 256 ? 1 : 2, 8, 1><<<grid, block, 0, st>>>(a);
  if (pl.waves == 4 && pl.groups == 1) pr_kernel<Tv, DP, 1, 4, 1><<<grid, block, 0, st>>>(a);
  if constexpr (sizeof(Tv) == 2 || DP == 64)
    if (pl.groups == 2) pr_kernel<Tv, DP, 1, 4, 2><<<grid, block, 0, st>>>(a);
  if constexpr (sizeof(Tv) == 2 && DP <= 128)
    if (pl.groups == 4) pr_kernel<Tv, DP, 1, 4, 4><<<grid, block, 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv>
int pr_run(const PrArgs& a, const PrPlan& pl, hipStream_t st) {
  const int rc = pl.dp == 64 ? pr_launch<Tv, 64>(a, pl, st)
               : pl.dp == 128 ? pr_launch<Tv, 128>(a, pl, st)
                              : pr_launch<Tv, 256>(a, pl, st);
  if (rc != MOE_OK || a.splits == 1) return rc;
  const JoinArgs jn = {a.part_o, a.part_ml, a.q_offsets, a.B + 1, a.N * a.Hq, a.Hq, a.D, a.splits,
                       a.out, a.lse};
  return attention_join<Tv>(jn, st);
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_prompt_attention_workspace(int64_t N, int64_t M, int64_t B, int32_t Hq,
                                                 int32_t Hkv, int32_t D, int32_t dtype) {
  using namespace moe;
  if (!pr_ok(N, M, B, Hq, Hkv, D, dtype) || !pr_supported(N, M, B, Hq, Hkv, D)) return 0;
  return pr_plan(N, M, B, Hq, Hkv, D, dtype).total;
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
  const PrPlan pl = pr_plan(N, M, B, Hq, Hkv, D, dtype);
  const Span in[] = {span_rows(q, N, q_stride * elt, Hq * D * elt),
                     span_rows(k, M, k_stride * elt, Hkv * D * elt),
                     span_rows(v, M, v_stride * elt, Hkv * D * elt),
                     {q_offsets, (B + 1) * 4}, {k_offsets, (B + 1) * 4}};
  const Span outs[] = {{out, N * Hq * D * elt}, {lse, N * Hq * 4},
                       {workspace, pl.splits > 1 ? (int64_t)pl.total : 0}};
  MOE_CHECK_ARG(spans_apart(outs, in));
  if (pl.splits > 1 &&
      (!workspace || ws_bytes < pl.total || (reinterpret_cast<uintptr_t>(workspace) & 255)))
    return MOE_ERR_WORKSPACE;
  const ScoreScale sc = score_scale(scale, dtype == MOE_BF16);
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
  a.nq = Hq / Hkv;
  a.per_nq = 1.f / (float)a.nq;
  a.scale2 = sc.scale2;
  a.keep = sc.keep;
  a.flip = sc.flip;
  a.splits = pl.splits;
  a.slots = pl.slots;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + pl.ml);
  a.out = out;
  a.lse = lse;
  hipStream_t st = as_stream(stream);
  return dtype == MOE_BF16 ? pr_run<uint16_t>(a, pl, st) : pr_run<float>(a, pl, st);
}
