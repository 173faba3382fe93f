// moe_beam_select and moe_beam_reorder: the choice of a request's best
// continuations, and the beams' states following it.
//
// Selection is one pass over the logits, which bounds it (HBM). c(b, v) =
// score_b + z_bv - lse_b ranks a row's tokens by their logits alone, so a block
// takes a chunk of one row into registers once and leaves the n best of it by
// logit with its share of the row's log-sum-exp; a second launch, one block a
// request, adds up the shares and merges the lists.
// Keys are (value, index) pairs, larger value first, lower index among equal
// values: no two are equal, which bounds how many can lie above a threshold
// whatever the logits hold.
#include "moeflow_decode.h"
#include "common.h"
#include "buffers.h"

#include <algorithm>

namespace moe {
namespace {

constexpr int kSelThreads = 256;
constexpr int kSelWaves = kSelThreads / kWave;
constexpr int kSelMaxBeams = 32, kSelMaxOut = 64;
constexpr int kSelChunk = 8192;                  // largest chunk of a row
constexpr int kMergeThreads = 512;
constexpr int kMergeLists = 4096 + kSelMaxBeams; // K * ceil(V / 8192) for K * V <= 2^25

struct SelLayout {
  size_t stat, val, idx, total;
  int64_t chunks;
  int ept;                                       // logits a thread takes
};

// Elements of a thread: 32, or 8 while the grid of the larger chunks would leave
// compute units idle.
SelLayout sel_layout(int64_t B, int32_t K, int64_t V, int32_t n_out) {
  SelLayout s{};
  s.ept = B * K * ceil_div(V, kSelChunk) < 256 && K * ceil_div(V, kSelChunk / 4) <= kMergeLists ? 8 : 32;
  s.chunks = ceil_div(V, (int64_t)s.ept * kSelThreads);
  const size_t lists = (size_t)(B * K * s.chunks);
  size_t o = 0;
  s.stat = o;                                    // {max, sum} of a chunk, double
  o = align_up(o + lists * 16, 256);
  s.val = o;                                     // the chunk's best logits, descending
  o = align_up(o + lists * n_out * 4, 256);
  s.idx = o;                                     // their tokens, -1 past the last
  o = align_up(o + lists * n_out * 4, 256);
  s.total = o;
  return s;
}

template <typename V>
__device__ __forceinline__ bool ahead(V a, int64_t ai, V b, int64_t bi) {
  return a > b || (a == b && ai < bi);
}

__device__ __forceinline__ float wave_max(float v) {
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
  return v;
}

__device__ __forceinline__ int wave_min(int v) {
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, kWave));
  return v;
}

// 16 bytes from an address that is only element-aligned.
struct __attribute__((packed, aligned(2))) Bytes16 { uint32_t w[4]; };

template <typename Tv> struct LogitVec;
template <> struct LogitVec<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const uint16_t* p, float* out) {
    const Bytes16 b = *reinterpret_cast<const Bytes16*>(p);
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
  static __device__ __forceinline__ void load(const float* p, float* out) {
    const Bytes16 b = *reinterpret_cast<const Bytes16*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = __uint_as_float(b.w[i]);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};

// One block: logits [c0, c0 + chunk) of row r in registers.
//   1. chunk maximum and sum of exp (float32 terms, at most EPT of them added in
//      float32, the rest in float64);
//   2. per wave, the n-th largest of its lanes' best keys; the largest of these
//      over the waves is a lower bound T of the chunk's n-th key, and at most
//      n lanes of a wave hold keys from T on;
//   3. keys from T on go to LDS (at most n * EPT a wave) and the n best of them
//      are ranked by counting.
template <typename Tv, int EPT>
__global__ void __launch_bounds__(kSelThreads)
beam_rows_kernel(const Tv* __restrict__ logits, int64_t V, const int32_t* __restrict__ finished,
                 int n, double2* __restrict__ stat, float* __restrict__ out_val,
                 int32_t* __restrict__ out_idx) {
  using LV = LogitVec<Tv>;
  constexpr int VE = LV::N, NV = EPT / VE;
  extern __shared__ float s_val[];               // n * EPT * waves values, then as many tokens
  int32_t* const s_idx = reinterpret_cast<int32_t*>(s_val + (size_t)n * EPT * kSelWaves);
  __shared__ float w_max[kSelWaves], w_thr[kSelWaves];
  __shared__ int w_thr_idx[kSelWaves];
  __shared__ double w_sum[kSelWaves];
  __shared__ int s_count;
  const int64_t row = blockIdx.y;
  const int64_t list = row * gridDim.x + blockIdx.x;
  if (finished && finished[row] != 0) return;    // its list is not read
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int64_t c0 = (int64_t)blockIdx.x * EPT * kSelThreads;
  const Tv* const base = logits + row * V;
  float z[EPT];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t at = c0 + ((int64_t)j * kSelThreads + threadIdx.x) * VE;
    if (at + VE <= V) {
      LV::load(base + at, z + j * VE);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) z[j * VE + i] = at + i < V ? LV::one(base + at + i) : -INFINITY;
    }
  }
  auto token = [&](int e) {                      // of register e: below 2^25
    return (int)(c0 + ((int64_t)(e / VE) * kSelThreads + threadIdx.x) * VE + e % VE);
  };
  if (threadIdx.x == 0) s_count = 0;

  // the lane's best key: the first of its largest numbers (its tokens ascend)
  float best = -INFINITY;
#pragma unroll
  for (int e = 0; e < EPT; ++e) best = fmaxf(best, z[e]);
  int best_idx = 0x7fffffff;
#pragma unroll
  for (int e = EPT - 1; e >= 0; --e) best_idx = z[e] == best ? token(e) : best_idx;
  float m = wave_max(best);
  if (lane == 0) w_max[wave] = m;

  // n-th largest of the lanes' keys: n times the largest leaves
  float left = best, thr = -INFINITY;
  int thr_idx = 0x7fffffff;
  for (int j = 0; j < n; ++j) {
    const float top = j == 0 ? m : wave_max(left);
    thr = top;
    if (top == -INFINITY) break;
    uint64_t at = ballot(left == top);
    int first;
    if (at & (at - 1)) {                         // equal values: the lowest token
      first = wave_min(left == top ? best_idx : 0x7fffffff);
    } else {
      first = __builtin_amdgcn_readlane(best_idx, __ffsll((unsigned long long)at) - 1);
    }
    thr_idx = first;
    if (left == top && best_idx == first) left = -INFINITY;
  }
  if (lane == 0) {
    w_thr[wave] = thr;
    w_thr_idx[wave] = thr_idx;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) m = fmaxf(m, w_max[w]);
  thr = w_thr[0];
  thr_idx = w_thr_idx[0];
#pragma unroll
  for (int w = 1; w < kSelWaves; ++w)
    if (ahead(w_thr[w], w_thr_idx[w], thr, thr_idx)) {
      thr = w_thr[w];
      thr_idx = w_thr_idx[w];
    }

  // sum of exp(z - m); a chunk of -inf adds nothing, NaN and +inf make it NaN
  const float shift = m == -INFINITY ? 0.f : m;
  float part = 0.f;
#pragma unroll
  for (int e = 0; e < EPT; ++e)
    part += __builtin_amdgcn_exp2f((z[e] - shift) * 1.4426950408889634f);
  const double wsum = wave_sum((double)part);
  if (lane == 0) w_sum[wave] = wsum;

  const int cap = n * EPT * kSelWaves;
  if (best > thr || (best == thr && best_idx <= thr_idx)) {
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const bool in = z[e] > -INFINITY && (z[e] > thr || (z[e] == thr && token(e) <= thr_idx));
      if (in) {
        const int at = atomicAdd(&s_count, 1);
        if (at < cap) {
          s_val[at] = z[e];
          s_idx[at] = token(e);
        }
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = w_sum[0];
    for (int w = 1; w < kSelWaves; ++w) t += w_sum[w];
    stat[list] = make_double2((double)m, t);
  }
  const int c = min(s_count, cap);
  for (int q = threadIdx.x; q < c; q += kSelThreads) {
    const float v = s_val[q];
    const int i = s_idx[q];
    int rank = 0;
    for (int o = 0; o < c; ++o) rank += ahead(s_val[o], s_idx[o], v, i);
    if (rank < n) {
      out_val[list * n + rank] = v;
      out_idx[list * n + rank] = i;
    }
  }
  for (int q = c + threadIdx.x; q < n; q += kSelThreads) {
    out_val[list * n + q] = -INFINITY;
    out_idx[list * n + q] = -1;
  }
}

// One block per request: the rows' log-sum-exp, then the n best of the lists.
// The n-th largest of the lists' first keys is a lower bound of the n-th key,
// and fewer than n lists hold keys above it: at most n * n keys are ranked.
__global__ void __launch_bounds__(kMergeThreads)
beam_merge_kernel(int K, int64_t V, int chunks, int n, const float* __restrict__ scores,
                  const int32_t* __restrict__ finished, int64_t eos,
                  const double2* __restrict__ stat, const float* __restrict__ val,
                  const int32_t* __restrict__ idx, int32_t* __restrict__ parent,
                  int32_t* __restrict__ token, float* __restrict__ out_scores,
                  int32_t* __restrict__ out_finished) {
  __shared__ double s_key[kMergeLists];          // first keys, then the keys to rank
  __shared__ int32_t s_pos[kMergeLists];         // beam * V + token, below 2^25
  __shared__ double s_off[kSelMaxBeams];         // score - lse, or the score of a finished beam
  __shared__ int s_done[kSelMaxBeams];
  __shared__ double s_thr;
  __shared__ int s_thr_pos, s_count;
  const int64_t b = blockIdx.x;
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  if (threadIdx.x == 0) {
    s_thr = -INFINITY;
    s_thr_pos = 0x7fffffff;
    s_count = 0;
  }
  // a row's chunks are added lane by lane, then over the lanes: a fixed order
  for (int k = wave; k < K; k += kMergeThreads / kWave) {
    const int64_t row = b * K + k;
    const int done = finished && finished[row] != 0;
    double off = (double)scores[row];
    if (!done) {
      double m = -INFINITY, t = 0.0;
      for (int c = lane; c < chunks; c += kWave) m = fmax(m, stat[row * chunks + c].x);
      for (int o = 32; o > 0; o >>= 1) m = fmax(m, __shfl_xor(m, o, kWave));
      for (int c = lane; c < chunks; c += kWave) {
        const double2 s = stat[row * chunks + c];
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
  __syncthreads();
  const int lists = K * chunks;
  // key j of list l; the single key of a finished beam is in its first list
  auto key = [&](int l, int j, double& c, int32_t& pos) {
    const int k = l / chunks;
    c = -INFINITY;
    pos = 0x7fffffff;
    int64_t t = -1;
    if (s_done[k]) {
      if (l % chunks == 0 && j == 0) {
        c = s_off[k];
        t = eos;
      }
    } else {
      const int64_t at = ((b * K) * chunks + l) * n + j;
      t = idx[at];
      if (t >= 0) c = (double)val[at] + s_off[k];
    }
    if (t < 0 || !(c > -INFINITY)) c = -INFINITY;          // NaN too
    else pos = (int32_t)(k * V + t);
  };
  for (int l = threadIdx.x; l < lists; l += kMergeThreads) {
    double c;
    int32_t pos;
    key(l, 0, c, pos);
    s_key[l] = c;
    s_pos[l] = pos;
  }
  __syncthreads();
  if (lists > n) {
    for (int l = threadIdx.x; l < lists; l += kMergeThreads) {
      const double c = s_key[l];
      const int32_t pos = s_pos[l];
      if (!(c > -INFINITY)) continue;
      int rank = 0;
      for (int o = 0; o < lists; ++o) rank += ahead(s_key[o], s_pos[o], c, pos);
      if (rank == n - 1) {                       // at most one list
        s_thr = c;
        s_thr_pos = pos;
      }
    }
  }
  __syncthreads();
  const double thr = s_thr;
  const int32_t thr_pos = s_thr_pos;
  // lists of at most n, and at most n of them reach the threshold
  for (int q = threadIdx.x; q < lists * n; q += kMergeThreads) {
    double c;
    int32_t pos;
    key(q / n, q % n, c, pos);
    if (c > -INFINITY && (c > thr || (c == thr && pos <= thr_pos))) {
      const int at = atomicAdd(&s_count, 1);
      if (at < kMergeLists) {
        s_key[at] = c;
        s_pos[at] = pos;
      }
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
  for (int q = threadIdx.x; q < count; q += kMergeThreads) {
    const double c = s_key[q];
    const int32_t pos = s_pos[q];
    int rank = 0;
    for (int o = 0; o < count; ++o) rank += ahead(s_key[o], s_pos[o], c, pos);
    if (rank < n) {
      const int k = (int)(pos / V);
      const int32_t t = (int32_t)(pos % V);
      put(rank, (int32_t)(b * K + k), t, (float)c, t == eos || s_done[k]);
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
  return K <= kSelMaxBeams && n_out <= kSelMaxOut && V <= ((int64_t)1 << 25) / K &&
         B < ((int64_t)1 << 31) / 64 / K;
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
  const SelLayout lay = sel_layout(B, K, V, n_out);
  if (!workspace || ws_bytes < lay.total || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return MOE_ERR_WORKSPACE;
  char* const ws = static_cast<char*>(workspace);
  hipStream_t st = as_stream(stream);
  auto* stat = reinterpret_cast<double2*>(ws + lay.stat);
  auto* val = reinterpret_cast<float*>(ws + lay.val);
  auto* idx = reinterpret_cast<int32_t*>(ws + lay.idx);
  const unsigned lds = (unsigned)(n_out * lay.ept * kSelWaves * 8);
  // rows in slices of the y dimension's limit
  constexpr int64_t kSlice = 32768;
  for (int64_t r0 = 0; r0 < B * K; r0 += kSlice) {
    const dim3 grid((unsigned)lay.chunks, (unsigned)std::min<int64_t>(kSlice, B * K - r0));
    const int32_t* const fin = finished ? finished + r0 : nullptr;
    const int64_t l0 = r0 * lay.chunks;
#define MOE_ROWS(T, EPT)                                                                   \
  beam_rows_kernel<T, EPT><<<grid, dim3(kSelThreads), lds, st>>>(                          \
      static_cast<const T*>(logits) + r0 * V, V, fin, n_out, stat + l0, val + l0 * n_out,  \
      idx + l0 * n_out)
    if (dtype == MOE_BF16) {
      if (lay.ept == 8) MOE_ROWS(uint16_t, 8);
      else MOE_ROWS(uint16_t, 32);
    } else {
      if (lay.ept == 8) MOE_ROWS(float, 8);
      else MOE_ROWS(float, 32);
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
  MOE_CHECK_ARG(!new_lens || new_lens != lens);
  if (K > kSelMaxBeams || B >= ((int64_t)1 << 31) / K || unit_bytes >= ((int64_t)1 << 31) ||
      S >= ((int64_t)1 << 31) / unit_bytes)      // 32-bit offsets within a row
    return MOE_ERR_UNSUPPORTED;
  // bytes of a cache stay below 2^62
  const double bytes = (double)L * (double)B * K * ((double)S + 1.0) * (double)unit_bytes;
  if (bytes > 4e18) return MOE_ERR_UNSUPPORTED;
  ReCaches c{};
  uintptr_t low = (uintptr_t)unit_bytes;         // common alignment of every row
  for (int32_t i = 0; i < n_caches; ++i) {
    if (S == 0) continue;                        // no bytes: only new_lens is written
    MOE_CHECK_ARG(caches[i]);
    for (int32_t j = 0; j < i; ++j) MOE_CHECK_ARG(caches[i] != caches[j]);
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
