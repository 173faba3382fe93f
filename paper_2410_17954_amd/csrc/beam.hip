// moe_beam_select and moe_beam_reorder: the choice of a request's best
// continuations, and the beams' states following it.
//
// Selection is one pass over the logits. c(b, v) = score_b + z_bv - lse_b ranks a
// row's tokens by their logits alone, so a block takes a chunk of one row into
// registers once and leaves the n best of it by logit with its share of the row's
// log-sum-exp; a second launch, one block a request, adds up the shares and merges
// the lists.
// Keys are (value, index) pairs, larger value first, lower index among equal
// values: no two are equal, which bounds how many can lie above a threshold
// whatever the logits hold. A merge's index is the beam, then the logit, larger
// first, then the token: beside a large score float64 sums of different logits are
// equal, and only with the logit in it is the order that of the chunks' lists.
#include "moeflow_decode.h"
#include "common.h"
#include "buffers.h"
#include "rows.h"

#include <float.h>

#include <algorithm>

namespace moe {
namespace {

constexpr int kSelThreads = 256;
constexpr int kSelWaves = kSelThreads / kWave;
constexpr int kSelMaxBeams = 32, kSelMaxOut = 64;
constexpr int kMergeThreads = 512;
constexpr int kMergeCopy = 4096;                 // keys that a merge keeps in LDS
constexpr int kMergeLists = 4096 + kSelMaxBeams; // lists of a request, keys that reach a threshold
constexpr uint64_t kNoPos = ~0ull;               // behind every key

// Of a merge: a continuation's sum and its place, beam << 57 | logit << 25 | token in
// their order, which decides between equal sums. 16 bytes, one LDS read.
struct alignas(16) SelKey { double c; uint64_t pos; };

struct SelLayout {
  size_t stat, val, idx, total;
  int64_t chunks;                                // of a row, a block each
  int ept;                                       // logits a thread takes
};

// 64, or 8 while longer chunks would leave compute units idle: K times the short
// chunks are then below 8 * 256, lists that a merge can take. Small calls have more
// chunks than larger ones for it, so `total` allows every call for as many as any of
// fewer requests, beams or tokens has, and never falls as a call grows.
SelLayout sel_layout(int64_t B, int32_t K, int64_t V, int32_t n_out) {
  constexpr int64_t kIdle = 256;
  static_assert(8 * kIdle <= kMergeLists, "short chunks of a request");
  SelLayout s{};
  const int64_t n64 = ceil_div(V, kSelThreads * 64), n8 = ceil_div(V, kSelThreads * 8);
  s.ept = B * K * n64 < kIdle ? 8 : 64;
  s.chunks = s.ept == 8 ? n8 : n64;
  auto take = [&](size_t lists) {
    size_t o = 0;
    s.stat = o;                                  // {ref, sum of exp(z - ref)} of a chunk, double
    o = align_up(o + lists * 16, 256);
    s.val = o;                                   // the chunk's best logits, descending
    o = align_up(o + lists * n_out * 4, 256);
    s.idx = o;                                   // their tokens, -1 past the last
    return align_up(o + lists * n_out * 4, 256);
  };
  s.total = take((size_t)std::max(B * K * n64, std::min(B * K * n8, 8 * (kIdle - 1))));
  take((size_t)(B * K * s.chunks));
  return s;
}

template <typename V, typename I>
__device__ __forceinline__ bool ahead(V a, I ai, V b, I bi) {
  return (a > b) | ((a == b) & (ai < bi));       // no branch, behind which a load would wait
}

// 16 bytes from an address that is only element-aligned.
struct __attribute__((packed, aligned(2))) Bytes16 { uint32_t w[4]; };

template <typename Tv> struct LogitVec;
template <> struct LogitVec<uint16_t> {
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
template <> struct LogitVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const Bytes16& b, float* out) {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = __uint_as_float(b.w[i]);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};

// Over a wave: m, the largest value; t, the smallest of the largest values of
// groups of 2^g neighbouring lanes.
__device__ __forceinline__ void group_extremes(float v, int g, float& m, float& t) {
  m = t = v;
  auto step = [&](float om, float ot, int level) {
    m = fmaxf(m, om);
    t = level < g ? m : fminf(t, ot);
  };
  step(dpp<0xB1>(m), dpp<0xB1>(t), 0);
  step(dpp<0x4E>(m), dpp<0x4E>(t), 1);
  step(dpp<0x141>(m), dpp<0x141>(t), 2);
  step(dpp<0x140>(m), dpp<0x140>(t), 3);
  step(__shfl_xor(m, 16, kWave), __shfl_xor(t, 16, kWave), 4);
  step(__shfl_xor(m, 32, kWave), __shfl_xor(t, 32, kWave), 5);
}

// One block: a chunk of a row in registers.
//   1. T, the smallest of the largest logits of at least n groups of lanes (4 to
//      64 of them): a lower bound of the chunk's n-th logit, since every group
//      holds one from T on;
//   2. sum of exp (float32 terms, at most 32 of them added in float32, the rest
//      in float64);
//   3. logits from T on, some three times n of a chunk whose groups all hold logits,
//      go to LDS and are ranked by counting.
// Where a wave holds more than kSelPart of them (equal logits, sorted ones, or a
// row's last chunk that leaves a group without any: its largest is -inf, and every
// logit is from T on), n rounds over the registers pick the best after the one before
// instead. Such a last chunk decides a call of few rows: one request of 8 beams, n 64,
// over 8000 logits takes 362 us, of 4 beams, n 4, over 32000 bf16 ones 13.5, over
// 32000 float32 ones, whose chunks are all full enough, 10.2.
// 64 requests of 8 beams over 128000 bf16 logits (131 MB) take 39 us, 34 where the
// last-level cache holds them: the loads and the maxima 19, the sums 2, the
// candidates 6, the ranks 11. Blocks that start together load together, so what
// follows the loads is not hidden behind them, and long chunks have less of it (of
// 8192 logits 63 us, of 16384 54, both before the ranks lost their branches; blocks
// that walk over several with the next one's loads in flight were slower).
constexpr int kSelPart = 128;

template <typename Tv, int EPT>
__global__ void __launch_bounds__(kSelThreads, EPT == 64 ? 4 : 8)
beam_rows_kernel(const Tv* __restrict__ logits, int64_t V, const int32_t* __restrict__ finished,
                 int n, int group, double2* __restrict__ stat, float* __restrict__ out_val,
                 int32_t* __restrict__ out_idx) {
  using LV = LogitVec<Tv>;
  constexpr int VE = LV::N, NV = EPT / VE;
  __shared__ float s_val[kSelWaves * kSelPart];
  __shared__ int32_t s_idx[kSelWaves * kSelPart];
  __shared__ float w_max[kSelWaves], w_thr[kSelWaves];
  __shared__ double w_sum[kSelWaves];
  __shared__ float w_best[kSelWaves];
  __shared__ int32_t w_idx[kSelWaves], w_count[kSelWaves];
  const int64_t row = blockIdx.y;
  if (finished && finished[row] != 0) return;    // its lists are not read
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // register e: token c0 + place(e) of the chunk at c0, below 2^25
  auto place = [&](int e) { return ((e / VE) * kSelThreads + (int)threadIdx.x) * VE + e % VE; };
  const int64_t list = row * gridDim.x + blockIdx.x;
  const int64_t c0 = (int64_t)blockIdx.x * EPT * kSelThreads;
  const int left = (int)min(V - c0, (int64_t)EPT * kSelThreads);
  const Tv* const base = logits + row * V + c0;
  float z[EPT];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = place(j * VE);
    Bytes16 raw = {};
    if (at + VE <= left) raw = *reinterpret_cast<const Bytes16*>(base + at);
    LV::unpack(raw, z + j * VE);
  }
  if (left < EPT * kSelThreads) {                // the row's end: at most one vector is cut
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = place(j * VE);
      if (at + VE > left)
#pragma unroll
        for (int i = 0; i < VE; ++i) z[j * VE + i] = -INFINITY;
      if (at < left && at + VE > left) {
#pragma unroll
        for (int i = 0; i < VE - 1; ++i)
          if (at + i < left) z[j * VE + i] = LV::one(base + at + i);
      }
    }
  }
  float best = -INFINITY;                        // a NaN is no maximum
#pragma unroll
  for (int e = 0; e < EPT; ++e) best = fmaxf(best, z[e]);
  float m, thr;
  group_extremes(best, group, m, thr);
  if (lane == 0) {
    w_max[wave] = m;
    w_thr[wave] = thr;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    m = fmaxf(m, w_max[w]);
    thr = fminf(thr, w_thr[w]);
  }

  // sum of exp(z - m) as 2^(z L - m L): one fma, whose rounding is that of the
  // small result; m L is rounded first and L is log2 e rounded, so what is summed
  // is exp(z - ref) up to (z - m) (1 - ln 2 L), with ref below. Where m L overflows
  // (masks of the lowest number) and for a chunk of -inf, which adds nothing, the
  // difference is taken first; NaN and +inf make the sum NaN.
  constexpr float L = 1.4426950408889634f;
  constexpr int PART = EPT < 32 ? EPT : 32;
  const bool plain = !(fabsf(m) < 1e38f);
  const float shift = plain ? (m == -INFINITY ? 0.f : m) : m * L;
  double dsum = 0.0;
#pragma unroll
  for (int e0 = 0; e0 < EPT; e0 += PART) {
    float part = 0.f;
    if (plain) {
#pragma unroll
      for (int e = e0; e < e0 + PART; ++e) part += __builtin_amdgcn_exp2f((z[e] - shift) * L);
    } else {
#pragma unroll
      for (int e = e0; e < e0 + PART; ++e) part += __builtin_amdgcn_exp2f(fmaf(z[e], L, -shift));
    }
    dsum += (double)part;
  }
  dsum = wave_sum(dsum);
  if (lane == 0) w_sum[wave] = dsum;

  thr = fmaxf(thr, -FLT_MAX);                    // -inf is no candidate
  float* const mine = s_val + wave * kSelPart;
  int32_t* const mine_idx = s_idx + wave * kSelPart;
  int found = 0;                                 // the wave's, all of them
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    const uint64_t in = ballot(z[e] >= thr);
    if (in == 0) continue;
    const int at = found + __popcll(in & lanemask_lt());
    if (z[e] >= thr && at < kSelPart) {
      mine[at] = z[e];
      mine_idx[at] = place(e);
    }
    found += __popcll(in);
  }
  if (lane == 0) w_count[wave] = found;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = w_sum[0];
    for (int w = 1; w < kSelWaves; ++w) t += w_sum[w];
    // 2^(m L - shift) = exp(m - ref)
    const double ref = (double)m + ((double)shift - (double)m * (double)L) * 0.6931471805599453;
    stat[list] = make_double2(plain ? (double)m : ref, t);
  }
  float* const val = out_val + list * n;
  int32_t* const idx = out_idx + list * n;
  int most = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    most = max(most, w_count[w]);
    total += w_count[w];
  }
  if (most <= kSelPart) {
    // a wave's keys against all: lanes 4 apart share a key, a wave's part each
    for (int q0 = 0; q0 < found; q0 += kWave / kSelWaves) {
      const int q = q0 + lane / kSelWaves, w = lane % kSelWaves;
      const bool ok = q < found;
      const float v = ok ? mine[q] : 0.f;
      const int i = ok ? mine_idx[q] : 0;
      const int end = ok ? w_count[w] : 0;
      int r = 0;
#pragma unroll 4
      for (int o = 0; o < end; ++o) r += ahead(s_val[w * kSelPart + o], s_idx[w * kSelPart + o], v, i);
      r += dpp<0xB1>(r);
      r += dpp<0x4E>(r);
      if (ok && w == 0 && r < n) {
        val[r] = v;
        idx[r] = (int)c0 + i;
      }
    }
    for (int q = total + threadIdx.x; q < n; q += kSelThreads) {
      val[q] = -INFINITY;
      idx[q] = -1;
    }
    return;
  }
  float pv = INFINITY;                           // the key before: everything comes after it
  int pi = -1;
  for (int j = 0; j < n; ++j) {                  // more than n numbers: there is always one left
    float bv = -INFINITY;
    int bi = 0x7fffffff;
    int at0 = (int)threadIdx.x * VE;             // opaque, or all places live in registers
    asm volatile("" : "+v"(at0));
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const int at = at0 + (e / VE) * kSelThreads * VE + e % VE;
      // a lane's places ascend: the first of its largest stays
      const bool after = z[e] < pv || (z[e] == pv && at > pi);
      if (after && (z[e] > bv || bi == 0x7fffffff)) {
        bv = z[e];
        bi = at;
      }
    }
    for (int o = 32; o > 0; o >>= 1) {
      const float ov = __shfl_xor(bv, o, kWave);
      const int oi = __shfl_xor(bi, o, kWave);
      if (ahead(ov, oi, bv, bi)) {
        bv = ov;
        bi = oi;
      }
    }
    if (lane == 0) {
      w_best[wave] = bv;
      w_idx[wave] = bi;
    }
    __syncthreads();
    pv = w_best[0];
    pi = w_idx[0];
#pragma unroll
    for (int w = 1; w < kSelWaves; ++w)
      if (ahead(w_best[w], w_idx[w], pv, pi)) {
        pv = w_best[w];
        pi = w_idx[w];
      }
    if (threadIdx.x == 0) {
      val[j] = pv;
      idx[j] = (int)c0 + pi;
    }
    __syncthreads();                             // w_best is rewritten next
  }
}

// rank[i] = keys ahead of key i, for i < count, by the whole block: as many threads
// share a key as there are. rank is zero on entry; ends with a barrier.
__device__ __forceinline__ void merge_ranks(const SelKey* key, int count, int32_t* rank) {
  const int per = max(1, kMergeThreads / max(count, 1));
  for (int q = threadIdx.x; q < count * per; q += kMergeThreads) {
    const int i = q % count, p = q / count;
    const SelKey mine = key[i];
    int r = 0;
#pragma unroll 4
    for (int o = count * p / per; o < count * (p + 1) / per; ++o) {
      const SelKey k = key[o];
      r += ahead(k.c, k.pos, mine.c, mine.pos);
    }
    if (r) atomicAdd(&rank[i], r);
  }
  __syncthreads();
}

// One block per request: the rows' log-sum-exp, then the n best of the lists.
// The n-th largest of the lists' first keys is a lower bound of the n-th key,
// and fewer than n lists hold keys above it: at most n * n keys are ranked. Such
// a block is bound by its loads' latency: the lists go to LDS beside the rows'
// sums where they fit.
__global__ void __launch_bounds__(kMergeThreads)
beam_merge_kernel(int K, int64_t V, int chunks, int n, const float* scores,
                  const int32_t* finished, int64_t eos,
                  const double2* __restrict__ stat, const float* __restrict__ val,
                  const int32_t* __restrict__ idx, int32_t* __restrict__ parent,
                  int32_t* __restrict__ token, float* out_scores,
                  int32_t* out_finished) {
  __shared__ SelKey s_key[kMergeLists];          // first keys, then the keys to rank
  __shared__ int32_t s_rank[kMergeLists];
  __shared__ float c_val[kMergeCopy];
  __shared__ int32_t c_idx[kMergeCopy];
  __shared__ double s_off[kSelMaxBeams];         // score - lse, or the score of a finished beam
  __shared__ int s_done[kSelMaxBeams];
  __shared__ SelKey s_thr;
  __shared__ int s_count;
  const int64_t b = blockIdx.x;
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int lists = K * chunks, keys = lists * n;
  const float* const g_val = val + b * keys;
  const int32_t* const g_idx = idx + b * keys;
  const bool copied = keys <= kMergeCopy;
  float fv[kMergeCopy / kMergeThreads];
  int32_t fi[kMergeCopy / kMergeThreads];
  if (copied) {
#pragma unroll
    for (int i = 0; i < kMergeCopy / kMergeThreads; ++i) {
      const int q = threadIdx.x + i * kMergeThreads;
      fv[i] = q < keys ? g_val[q] : 0.f;
      fi[i] = q < keys ? g_idx[q] : -1;
    }
  }
  if (threadIdx.x == 0) {
    s_thr = SelKey{-INFINITY, kNoPos};
    s_count = 0;
  }
  for (int l = threadIdx.x; l < kMergeLists; l += kMergeThreads) s_rank[l] = 0;
  // a row's chunks are added lane by lane, then over the lanes: a fixed order
  for (int k = wave; k < K; k += kMergeThreads / kWave) {
    const int64_t row = b * K + k;
    const double2* const st = stat + row * chunks;
    double2 first = make_double2(-INFINITY, 0.0);
    if (lane < chunks) first = st[lane];
    const int done = finished && finished[row] != 0;
    double off = (double)scores[row];
    if (!done) {
      double m = first.x, t = 0.0;
      for (int c = lane + kWave; c < chunks; c += kWave) m = fmax(m, st[c].x);
      for (int o = 32; o > 0; o >>= 1) m = fmax(m, __shfl_xor(m, o, kWave));
      for (int c = lane; c < chunks; c += kWave) {
        const double2 s = c == lane ? first : st[c];
        t += s.x == -INFINITY ? s.y : s.y * exp(s.x - m);   // 0, or the NaN it holds
      }
      t = wave_sum(t);
      off -= m + log(t);
    }
    if (lane == 0) {
      s_off[k] = off;
      s_done[k] = done;
    }
  }
  if (copied) {
#pragma unroll
    for (int i = 0; i < kMergeCopy / kMergeThreads; ++i) {
      const int q = threadIdx.x + i * kMergeThreads;
      if (q < keys) {
        c_val[q] = fv[i];
        c_idx[q] = fi[i];
      }
    }
  }
  __syncthreads();
  // key j of list l of beam k; the single key of a finished beam is in its first list
  auto key = [&](int k, int l, int j) {
    double c = -INFINITY;
    int t = -1;
    float z = 0.f;                               // a finished beam has one key
    if (s_done[k]) {
      if (l == k * chunks && j == 0) {
        c = s_off[k];
        t = (int)eos;
      }
    } else {
      const int at = l * n + j;
      t = copied ? c_idx[at] : g_idx[at];
      if (t >= 0) {
        z = copied ? c_val[at] : g_val[at];
        c = (double)z + s_off[k];
      }
    }
    if (t < 0 || !(c > -INFINITY)) return SelKey{-INFINITY, kNoPos};   // NaN too
    return SelKey{c, (uint64_t)k << 57 | (uint64_t)~float_order(z) << 25 | (uint32_t)t};
  };
  for (int l = threadIdx.x; l < lists; l += kMergeThreads) s_key[l] = key(l / chunks, l, 0);
  __syncthreads();
  if (lists > n) {
    merge_ranks(s_key, lists, s_rank);
    for (int l = threadIdx.x; l < lists; l += kMergeThreads)
      if (s_rank[l] == n - 1 && s_key[l].c > -INFINITY) s_thr = s_key[l];   // at most one list
    __syncthreads();
    for (int l = threadIdx.x; l < lists; l += kMergeThreads) s_rank[l] = 0;
  }
  const SelKey thr = s_thr;
  // lists of at most n, in descending order, and at most n of them reach the threshold
  for (int l = threadIdx.x; l < lists; l += kMergeThreads) {
    const int k = l / chunks;
    for (int j = 0; j < n; ++j) {
      const SelKey c = key(k, l, j);
      if (!(c.c > -INFINITY) || ahead(thr.c, thr.pos, c.c, c.pos)) break;
      const int at = atomicAdd(&s_count, 1);
      if (at < kMergeLists) s_key[at] = c;
    }
  }
  __syncthreads();
  const int count = min(s_count, kMergeLists);
  auto put = [&](int at, int32_t row, int32_t t, float c, int fin) {
    parent[b * n + at] = row;
    token[b * n + at] = t;
    out_scores[b * n + at] = c;
    if (out_finished) out_finished[b * n + at] = fin;
  };
  merge_ranks(s_key, count, s_rank);
  for (int q = threadIdx.x; q < count; q += kMergeThreads) {
    const SelKey c = s_key[q];
    const int rank = s_rank[q];
    if (rank < n) {
      const int k = (int)(c.pos >> 57), t = (int)(c.pos & 0x1ffffff);
      put(rank, (int32_t)(b * K + k), t, (float)c.c, t == eos || s_done[k]);
    }
  }
  for (int q = count + threadIdx.x; q < n; q += kMergeThreads) put(q, -1, -1, -INFINITY, 0);
}

// ---------------------------------------------------------------- reorder
constexpr int kReThreads = 256, kReMaxCaches = 16;

struct ReCaches { char* base[kReMaxCaches]; };

// 16, 8, 4 or 1 bytes of a raw buffer per lane; past its end nothing is read
// (zeros) or written.
template <int ELT> struct Piece;
template <> struct Piece<16> {
  using T = u32x4_t;
  static __device__ __forceinline__ T load(rsrc_t r, int o) { return __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0); }
  static __device__ __forceinline__ void store(T v, rsrc_t r, int o) { __builtin_amdgcn_raw_buffer_store_b128(v, r, o, 0, 0); }
};
template <> struct Piece<8> {
  using T = __attribute__((ext_vector_type(2))) uint32_t;
  static __device__ __forceinline__ T load(rsrc_t r, int o) { return __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, 0); }
  static __device__ __forceinline__ void store(T v, rsrc_t r, int o) { __builtin_amdgcn_raw_buffer_store_b64(v, r, o, 0, 0); }
};
template <> struct Piece<4> {
  using T = uint32_t;
  static __device__ __forceinline__ T load(rsrc_t r, int o) { return __builtin_amdgcn_raw_buffer_load_b32(r, o, 0, 0); }
  static __device__ __forceinline__ void store(T v, rsrc_t r, int o) { __builtin_amdgcn_raw_buffer_store_b32(v, r, o, 0, 0); }
};
template <> struct Piece<1> {
  using T = uint8_t;
  static __device__ __forceinline__ T load(rsrc_t r, int o) { return __builtin_amdgcn_raw_buffer_load_b8(r, o, 0, 0); }
  static __device__ __forceinline__ void store(T v, rsrc_t r, int o) { __builtin_amdgcn_raw_buffer_store_b8(v, r, o, 0, 0); }
};

// A request's moves: row dst takes over len bytes of row src.
template <int MAXK>
struct Moves {
  int src[MAXK], dst[MAXK];
  uint32_t len[MAXK];                            // 0 past the last move
};

// The same bytes of M rows by one thread: it holds the sources of all of them in
// registers before it writes the first, so the move is in place whatever the
// parents are, and no thread waits for another.
template <int ELT, int M, int MAXK>
__device__ __forceinline__ void move_rows(char* rows, int64_t row_bytes, const Moves<MAXK>& mv,
                                          uint32_t longest) {
  auto rsrc = [&](int row, uint32_t len) {
    char* const p = rows + (int64_t)__builtin_amdgcn_readfirstlane(row) * row_bytes;
    return __builtin_amdgcn_make_buffer_rsrc(p, 0, __builtin_amdgcn_readfirstlane((int)len),
                                             0x00027000);
  };
  const uint32_t step = gridDim.x * kReThreads * ELT;
  for (uint32_t o = (blockIdx.x * kReThreads + threadIdx.x) * ELT; o < longest; o += step) {
    typename Piece<ELT>::T v[M];
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] = Piece<ELT>::load(rsrc(mv.src[i], mv.len[i]), (int)o);
#pragma unroll
    for (int i = 0; i < M; ++i) Piece<ELT>::store(v[i], rsrc(mv.dst[i], mv.len[i]), (int)o);
  }
}

// Block (x: pieces of a row, y: request, z: cache and layer). MAXK: the most
// beams (registers).
template <int ELT, int MAXK>
__global__ void __launch_bounds__(kReThreads)
beam_reorder_kernel(ReCaches caches, int n_caches, int64_t L, int64_t B, int K, int64_t S,
                    int64_t unit, const int32_t* __restrict__ parent,
                    const int32_t* __restrict__ lens, int32_t* __restrict__ new_lens,
                    int32_t* __restrict__ err) {
  __shared__ Moves<MAXK> mv;
  __shared__ int s_moves;
  const bool first = blockIdx.x == 0 && blockIdx.z == 0;
  for (int64_t b = blockIdx.y; b < B; b += gridDim.y) {
    __syncthreads();                             // the moves of the request before
    if (threadIdx.x == 0) s_moves = 0;
    if (threadIdx.x < MAXK) {
      mv.src[threadIdx.x] = mv.dst[threadIdx.x] = 0;
      mv.len[threadIdx.x] = 0;
    }
    __syncthreads();
    if (threadIdx.x < K) {
      const int r = threadIdx.x;
      const int64_t p = parent[b * K + r];
      const bool ok = p >= b * K && p < (b + 1) * K;
      if (first && !ok && p != -1) atomicExch(err, 1);
      const int src = ok ? (int)(p - b * K) : r;
      const int64_t len = lens ? min(max((int64_t)lens[b * K + src], (int64_t)0), S) : S;
      if (first && new_lens) new_lens[b * K + r] = lens ? lens[b * K + src] : (int32_t)S;
      if (src != r && len > 0) {
        const int at = atomicAdd(&s_moves, 1);
        mv.src[at] = src;
        mv.dst[at] = r;
        mv.len[at] = (uint32_t)(len * unit);     // below 2^31
      }
    }
    __syncthreads();
    // the same for the whole block, and known to be (scalar registers)
    const int moves = __builtin_amdgcn_readfirstlane(s_moves);
    uint32_t longest = 0;
    for (int i = 0; i < moves; ++i) longest = max(longest, mv.len[i]);
    for (int64_t cl = blockIdx.z; cl < L * n_caches; cl += gridDim.z) {
      const int64_t l = cl / n_caches;
      const int c = (int)(cl - l * n_caches);
      char* base = caches.base[0];
#pragma unroll
      for (int i = 1; i < kReMaxCaches; ++i) base = i == c ? caches.base[i] : base;
      char* const rows = base + (l * B + b) * K * S * unit;
      if (moves <= 1) move_rows<ELT, 1>(rows, S * unit, mv, longest);
      else if (moves <= 2) move_rows<ELT, 2>(rows, S * unit, mv, longest);
      else if (moves <= 4) move_rows<ELT, 4>(rows, S * unit, mv, longest);
      else if constexpr (MAXK >= 8) {
        if (moves <= 8) move_rows<ELT, 8>(rows, S * unit, mv, longest);
        else if constexpr (MAXK >= 32) {
          if (moves <= 16) move_rows<ELT, 16>(rows, S * unit, mv, longest);
          else move_rows<ELT, 32>(rows, S * unit, mv, longest);
        }
      }
    }
  }
}

bool sel_ok(int64_t B, int32_t K, int64_t V, int32_t n_out) {
  return B >= 1 && K >= 1 && V >= 1 && n_out >= 1;
}
bool sel_supported(int64_t B, int32_t K, int64_t V, int32_t n_out) {
  // a launch's dimension is below 2^32 threads: a merge block a request
  return K <= kSelMaxBeams && n_out <= kSelMaxOut && V <= ((int64_t)1 << 25) / K &&
         B < ((int64_t)1 << 31) / 64 / K && B < ((int64_t)1 << 32) / kMergeThreads;
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_beam_select_workspace(int64_t B, int32_t K, int64_t V, int32_t n_out) {
  if (!moe::sel_ok(B, K, V, n_out) || !moe::sel_supported(B, K, V, n_out)) return 0;
  return moe::sel_layout(B, K, V, n_out).total;
}

extern "C" int moe_beam_select(const void* logits, int32_t dtype, int64_t B, int32_t K, int64_t V,
                               const float* scores, const int32_t* finished, int64_t eos,
                               int32_t n_out, int32_t* parent, int32_t* token, float* out_scores,
                               int32_t* out_finished, void* workspace, size_t ws_bytes,
                               void* stream) {
  using namespace moe;
  MOE_CHECK_ARG(logits && scores && parent && token && out_scores);
  MOE_CHECK_ARG(valid_dtype(dtype) && sel_ok(B, K, V, n_out));
  MOE_CHECK_ARG((!finished && !out_finished) || (eos >= 0 && eos < V));
  const size_t elt = dtype == MOE_BF16 ? 2 : 4;
  MOE_CHECK_ARG(reinterpret_cast<uintptr_t>(logits) % elt == 0);
  if (!sel_supported(B, K, V, n_out)) return MOE_ERR_UNSUPPORTED;
  // in place a block would overwrite what another has yet to read
  MOE_CHECK_ARG(n_out == K || (out_scores != scores && (!finished || out_finished != finished)));
  const SelLayout lay = sel_layout(B, K, V, n_out);
  if (!workspace || ws_bytes < lay.total || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return MOE_ERR_WORKSPACE;
  char* const ws = static_cast<char*>(workspace);
  hipStream_t st = as_stream(stream);
  auto* stat = reinterpret_cast<double2*>(ws + lay.stat);
  auto* val = reinterpret_cast<float*>(ws + lay.val);
  auto* idx = reinterpret_cast<int32_t*>(ws + lay.idx);
  // lanes of a group, 2^group: 256 threads hold at least n_out groups
  int group = 6;
  while (group > 2 && (kSelThreads >> group) < n_out) --group;
  // rows in slices of the y dimension's limit
  constexpr int64_t kSlice = 32768;
  for (int64_t r0 = 0; r0 < B * K; r0 += kSlice) {
    const dim3 grid((unsigned)lay.chunks, (unsigned)std::min<int64_t>(kSlice, B * K - r0));
    const int32_t* const fin = finished ? finished + r0 : nullptr;
    const int64_t l0 = r0 * lay.chunks;
#define MOE_ROWS(T, EPT)                                                                         \
  beam_rows_kernel<T, EPT><<<grid, dim3(kSelThreads), 0, st>>>(                                  \
      static_cast<const T*>(logits) + r0 * V, V, fin, n_out, group, stat + l0, val + l0 * n_out, \
      idx + l0 * n_out)
    if (dtype == MOE_BF16) {
      if (lay.ept == 8) MOE_ROWS(uint16_t, 8);
      else MOE_ROWS(uint16_t, 64);
    } else {
      if (lay.ept == 8) MOE_ROWS(float, 8);
      else MOE_ROWS(float, 64);
    }
#undef MOE_ROWS
    MOE_CHECK_LAUNCH();
  }
  beam_merge_kernel<<<dim3((unsigned)B), dim3(kMergeThreads), 0, st>>>(
      K, V, (int)lay.chunks, n_out, scores, finished, eos, stat, val, idx, parent, token,
      out_scores, out_finished);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

extern "C" int moe_beam_reorder(void* const* caches, int32_t n_caches, int64_t L, int64_t B,
                                int32_t K, int64_t S, int64_t unit_bytes, const int32_t* parent,
                                const int32_t* lens, int32_t* new_lens, int32_t* err,
                                void* stream) {
  using namespace moe;
  MOE_CHECK_ARG(caches && parent && err);
  MOE_CHECK_ARG(n_caches >= 1 && n_caches <= kReMaxCaches && L >= 1 && B >= 1 && K >= 1 &&
                S >= 0 && unit_bytes >= 1);
  MOE_CHECK_ARG(!new_lens || (new_lens != lens && new_lens != parent));
  if (K > kSelMaxBeams || B >= ((int64_t)1 << 31) / K || unit_bytes >= ((int64_t)1 << 31) ||
      S >= ((int64_t)1 << 31) / unit_bytes)      // 32-bit offsets within a row
    return MOE_ERR_UNSUPPORTED;
  // bytes of a cache stay below 2^62
  const double bytes = (double)L * (double)B * K * ((double)S + 1.0) * (double)unit_bytes;
  if (bytes > 4e18) return MOE_ERR_UNSUPPORTED;
  const uintptr_t size = (uintptr_t)(L * B * K * S * unit_bytes);
  ReCaches c{};
  uintptr_t low = (uintptr_t)unit_bytes;         // common alignment of every row
  for (int32_t i = 0; i < n_caches; ++i) {
    if (S == 0) continue;                        // no bytes: only new_lens is written
    MOE_CHECK_ARG(caches[i]);
    const uintptr_t at = reinterpret_cast<uintptr_t>(caches[i]);
    for (int32_t j = 0; j < i; ++j) {            // blocks would read what others write
      const uintptr_t other = reinterpret_cast<uintptr_t>(caches[j]);
      MOE_CHECK_ARG(at + size <= other || other + size <= at);
    }
    c.base[i] = static_cast<char*>(caches[i]);
    low |= reinterpret_cast<uintptr_t>(caches[i]);
  }
  hipStream_t st = as_stream(stream);
  const int elt = low % 16 == 0 ? 16 : low % 8 == 0 ? 8 : low % 4 == 0 ? 4 : 1;
  const int64_t pieces = std::max<int64_t>(1, ceil_div(S * unit_bytes, kReThreads * elt));
  const dim3 grid((unsigned)std::min<int64_t>(pieces, 4096),
                  (unsigned)std::min<int64_t>(B, 4096),
                  (unsigned)std::min<int64_t>(L * n_caches, 4096));
#define MOE_RE(E, M)                                                                       \
  beam_reorder_kernel<E, M><<<grid, dim3(kReThreads), 0, st>>>(c, n_caches, L, B, K, S, unit_bytes, \
                                                               parent, lens, new_lens, err)
#define MOE_RE_K(E)           \
  do {                        \
    if (K <= 4) MOE_RE(E, 4); \
    else if (K <= 8) MOE_RE(E, 8); \
    else MOE_RE(E, 32);       \
  } while (0)
  if (elt == 16) MOE_RE_K(16);
  else if (elt == 8) MOE_RE_K(8);
  else if (elt == 4) MOE_RE_K(4);
  else MOE_RE_K(1);
#undef MOE_RE_K
#undef MOE_RE
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}
