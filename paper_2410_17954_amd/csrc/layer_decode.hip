// moe_layer_decode: a whole MoE layer (router, top-k gates, SwiGLU experts over
// the resident slots, shared experts, weighted sum) for at most 64 tokens.
//
// So few tokens leave the layer bound by reading the weights of the experts
// they reach once (HBM); the rest is launches and latencies, so there are three
// of the former (a fourth beyond 16 tokens) and no permuted copies:
//   ld_first_kernel  the router's logits in float64, spread over the chip
//   ld_up_kernel     blocks that stream the shared experts' gate and up rows; the
//                    others each decide the routes of all tokens for themselves
//                    (none needs another block), then stream the active experts'.
//                    They write
//                      a[t, :] = gate_t * silu(x_t . Wg^T) * (x_t . Wu^T)
//   ld_down_kernel   y[t, n] = sum over the experts of t of a . Wd[n, :]: the
//                    gates are in a, so the sums of all experts of a column
//                    tile run on in the same accumulators
// No block waits for another and nothing is added by atomics.
//
// A tile of weights is 16 rows, a K block the 128 bytes of a cache line of each
// (64 bf16 or 32 float32 values), loaded as two instructions of 8 rows x 128
// bytes (non-temporal: every byte is read once), whose halves lanes l and l ^ 8
// swap (see ror8_into). That leaves lane (row r, q) with the line's 16-byte
// chunks q and 4 + q, the operands of two K steps. Chunks past K and rows past
// the matrix lie past the end of the raw buffer or are sent there: zeros.
#include "moeflow_decode.h"
#include "common.h"
#include "buffers.h"
#include "rows.h"

#include <algorithm>
#include <type_traits>

namespace moe {
namespace {

constexpr int kLdTokens = 64, kLdMaxK = 32, kLdExperts = 256;
constexpr uint32_t kPastEnd = 0x7ffffff0u;       // no buffer here is as long

template <typename Tv> struct LdType;
template <> struct LdType<uint16_t> {
  static constexpr int KB = 64;                  // values per K block (128 bytes)
  static __device__ __forceinline__ void mfma(f32x4_t& c, const u32x4_t& a, const u32x4_t& w) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                __builtin_bit_cast(bf16x8_t, w), c, 0, 0, 0);
  }
  static __device__ __forceinline__ float act(float g, float u) { return swiglu(g, u); }
  static __device__ __forceinline__ uint16_t put(float v) { return f32_to_bf16(v); }
  static __device__ __forceinline__ float get(uint16_t v) { return bf16_to_f32(v); }
};
template <> struct LdType<float> {
  static constexpr int KB = 32;
  // the v-th value of every lane's chunk feeds the v-th MFMA: its four k are
  // four apart, the same for both operands
  static __device__ __forceinline__ void mfma(f32x4_t& c, const u32x4_t& a, const u32x4_t& w) {
#pragma unroll
    for (int v = 0; v < 4; ++v)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[v]), __uint_as_float(w[v]), c, 0,
                                               0, 0);
  }
  static __device__ __forceinline__ float act(float g, float u) { return g / (1.f + expf(-g)) * u; }
  static __device__ __forceinline__ float put(float v) { return v; }
  static __device__ __forceinline__ float get(float v) { return v; }
};

// An expert that tokens reached and that is resident: rows base .. base + rows
// of the activation, tokens ascending.
struct LdEntry {
  int32_t slot, base, rows;
};

struct LdLayout {
  size_t z, meta, entries, tokens, act, part, total;
};

int64_t act_rows_bytes(int64_t T, int32_t k, int64_t F, int64_t Fs, size_t elt) {
  return (int64_t)((size_t)T * k * F * elt + (size_t)T * Fs * elt);
}

// K parts of the down projection in blocks of 64 columns, two blocks for each of
// 256 compute units; 0: blocks of 16 or 8 columns, without parts. Up to 16 tokens
// the experts' rows are few, and so are the activation loads that wider blocks
// save (the launch, with the join where there are parts, us: 4 Mixtral-shaped
// tokens 112, in 64 columns 132; 7 Qwen-shaped 18, 32). Beyond, they weigh as much
// as the weights (32 Mixtral-shaped 177, in 64 columns 155; 64 Qwen-shaped 73, 46).
int ld_parts(int64_t T, int64_t H) {
  if (T <= 16) return 0;
  return (int)std::min<int64_t>(ceil_div(512, ceil_div(H, 64)), 16);
}

LdLayout ld_layout(int64_t T, int64_t H, int64_t F, int32_t E, int32_t k, int64_t Fs,
                   int32_t dtype) {
  const size_t elt = dtype == MOE_BF16 ? 2 : 4;
  LdLayout s{};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = align_up(o + bytes, 256);
    return at;
  };
  s.z = take((size_t)T * E * 8);
  s.meta = take(4);
  s.entries = take((size_t)E * sizeof(LdEntry));
  s.tokens = take((size_t)T * k);
  s.act = take((size_t)act_rows_bytes(T, k, F, Fs, elt));
  s.part = take((size_t)ld_parts(T, H) * T * H * 4);
  s.total = o;
  return s;
}

// ---------------------------------------------------------------- logits
// z[t, e] in float64 (bf16 products are exact in it), by one wave.
template <typename Tv>
__device__ __forceinline__ void ld_logit(const Tv* __restrict__ x, const Tv* __restrict__ wr, int t,
                                         int e, int64_t H, int E, const float* __restrict__ bias,
                                         int bias_mode, double* __restrict__ z) {
  constexpr int VE = 16 / sizeof(Tv);
  const int lane = lane_id();
  const Tv* const xr = x + (int64_t)t * H;
  const Tv* const w = wr + (int64_t)e * H;
  double a0 = 0.0, a1 = 0.0;
  auto dot = [&](const u32x4_t& xv, const u32x4_t& wv) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(Tv) == 2) {
        a0 = fma((double)__uint_as_float(xv[i] << 16), (double)__uint_as_float(wv[i] << 16), a0);
        a1 = fma((double)__uint_as_float(xv[i] & 0xffff0000u),
                 (double)__uint_as_float(wv[i] & 0xffff0000u), a1);
      } else {
        double& a = i & 1 ? a1 : a0;
        a = fma((double)__uint_as_float(xv[i]), (double)__uint_as_float(wv[i]), a);
      }
    }
  };
  constexpr int R = 4;
  int64_t h = (int64_t)lane * VE;
  for (; h + (R - 1) * kWave * VE < H; h += R * kWave * VE) {
    u32x4_t xv[R], wv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      xv[i] = *reinterpret_cast<const u32x4_t*>(xr + h + i * kWave * VE);
      wv[i] = *reinterpret_cast<const u32x4_t*>(w + h + i * kWave * VE);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) dot(xv[i], wv[i]);
  }
  for (; h < H; h += kWave * VE)
    dot(*reinterpret_cast<const u32x4_t*>(xr + h), *reinterpret_cast<const u32x4_t*>(w + h));
  double a = wave_sum(a0 + a1);
  if (lane == 0) {
    if (bias_mode == 1) a += (double)bias[e];
    if (bias_mode == 2) a += (double)bias[(int64_t)t * E + e];
    z[(int64_t)t * E + e] = a;
  }
}

// ---------------------------------------------------------------- routes
// What a block keeps of the routes of all tokens. TOK: tokens at most.
template <int TOK>
struct LdRoutes {
  static constexpr int PAIRS = TOK * kLdMaxK;
  uint64_t mask[kLdExperts];                     // tokens that chose a resident expert
  float gate[PAIRS];                             // by token and choice
  float row_gate[PAIRS];                         // by activation row
  float total[TOK];                              // sum of exp over all experts
  int32_t base[kLdExperts], slot[kLdExperts];
  int16_t sel[PAIRS];                            // expert of a choice, -1: none
  uint8_t row_token[PAIRS];
  uint8_t list[kLdExperts];                      // active experts, ascending
  int32_t wave_n[kLdExperts / kWave], wave_rows[kLdExperts / kWave];
  int32_t n_active;
};

__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
  v = max(v, (uint32_t)dpp<0xB1>((int)v));
  v = max(v, (uint32_t)dpp<0x4E>((int)v));
  v = max(v, (uint32_t)dpp<0x141>((int)v));
  return max(v, (uint32_t)dpp<0x140>((int)v));
}

// Top-k (larger logit, then lower expert; a NaN is never chosen nor part of the
// softmax; a token without a logit above -inf chooses nothing) of token t by
// the 16 lanes of a row; lane gl holds the logits of experts gl + 16 r. k rounds
// of row maximum over the logits' float32 roundings, whose order is that of the
// float64 logits wherever they differ; a round in which lanes of some row share
// the maximum is decided on the float64 values. Leaves ln of each choice's share
// of the largest exponential in s.gate.
template <int EPL, int TOK>
__device__ __forceinline__ void ld_decide(const double* __restrict__ z, bool live, int t, int E,
                                          int k, int renorm, int gl, LdRoutes<TOK>& s) {
  double v[EPL];
  uint32_t free = 0;
  double m = -INFINITY;
#pragma unroll
  for (int r = 0; r < EPL; ++r) {
    const int e = gl + kRowLanes * r;
    v[r] = live && e < E ? z[(int64_t)t * E + e] : -INFINITY;
    if (live && e < E && v[r] == v[r]) free |= 1u << r;
    m = fmax(m, v[r]);
  }
  m = fmax(m, dpp<0xB1>(m));
  m = fmax(m, dpp<0x4E>(m));
  m = fmax(m, dpp<0x141>(m));
  m = fmax(m, dpp<0x140>(m));
  if (m == -INFINITY) free = 0;                  // nothing above -inf: no choice
  if (!renorm) {
    float total = 0.f;
#pragma unroll
    for (int r = 0; r < EPL; ++r)
      if ((free >> r) & 1) total += expf((float)(v[r] - m));
    total += dpp<0xB1>(total);
    total += dpp<0x4E>(total);
    total += dpp<0x141>(total);
    total += dpp<0x140>(total);
    if (live && gl == 0) s.total[t] = total;
  }
  const uint32_t row_shift = (lane_id() / kRowLanes) * kRowLanes;
  for (int j = 0; j < k; ++j) {
    double bv = 0.0;
    int be = -1;
#pragma unroll
    for (int r = 0; r < EPL; ++r)
      if (((free >> r) & 1) && (be < 0 || v[r] > bv)) {
        bv = v[r];
        be = gl + kRowLanes * r;
      }
    const uint32_t key = be >= 0 ? float_order((float)bv) : 0u;   // 0 is no float's
    const uint32_t top = row_max_u32(key);
    const bool at_top = key == top && be >= 0;
    const uint32_t row = (uint32_t)(ballot(at_top) >> row_shift) & 0xffffu;
    bool won = at_top;
    if (ballot(live && (row & (row - 1)) != 0)) {
      double wv = bv;
      int we = be;
      row_argmax(wv, we);
      won = be >= 0 && we == be;
    }
    if (live && won) {
      s.sel[t * k + j] = (int16_t)be;
      s.gate[t * k + j] = (float)(bv - m);
      free &= ~(1u << (be / kRowLanes));
    }
    if (live && row == 0 && gl == 0) {           // no number left
      s.sel[t * k + j] = -1;
      s.gate[t * k + j] = -INFINITY;
    }
  }
}

// The routes of all tokens, by the whole block; ends with a barrier. Three
// dependent steps: logits, choices, lists.
template <int TOK, int THREADS>
__device__ __forceinline__ void ld_routes(const double* __restrict__ z, int T, int E, int k,
                                          int renorm, const int32_t* __restrict__ slot, int S,
                                          LdRoutes<TOK>& s) {
  static_assert(THREADS >= kLdExperts, "one thread per expert");
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int gl = lane % kRowLanes, grp = lane / kRowLanes;
  if (threadIdx.x < kLdExperts) {
    s.mask[threadIdx.x] = 0;
    const int sl = (int)threadIdx.x >= E ? -1 : slot ? slot[threadIdx.x] : (int)threadIdx.x;
    s.slot[threadIdx.x] = sl < S ? sl : -1;
  }
  for (int t0 = 0; t0 < T; t0 += THREADS / kRowLanes) {
    const int t = t0 + wave * (kWave / kRowLanes) + grp;
    const bool live = t < T;
    if (E <= 16) ld_decide<1>(z, live, live ? t : 0, E, k, renorm, gl, s);
    else if (E <= 64) ld_decide<4>(z, live, live ? t : 0, E, k, renorm, gl, s);
    else ld_decide<16>(z, live, live ? t : 0, E, k, renorm, gl, s);
  }
  __syncthreads();
  constexpr int Q = (LdRoutes<TOK>::PAIRS + THREADS - 1) / THREADS;
  float g[Q];
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    const int q = threadIdx.x + i * THREADS;
    if (q >= T * k) break;
    const int e = s.sel[q], t = q / k;
    if (e >= 0 && s.slot[e] >= 0)
      atomicOr(reinterpret_cast<unsigned long long*>(&s.mask[e]), 1ull << t);
    // float32 exponentials of float64 differences, their sum in choice order
    float den = 0.f;
    if (renorm)
      for (int j = 0; j < k; ++j) den += expf(s.gate[t * k + j]);
    else
      den = s.total[t];
    g[i] = e >= 0 ? expf(s.gate[q]) / den : 0.f;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    const int q = threadIdx.x + i * THREADS;
    if (q < T * k) s.gate[q] = g[i];
  }
  // one thread per expert: its place in the list and its first activation row
  const bool mine = threadIdx.x < kLdExperts;
  const int rows = mine ? __popcll(s.mask[threadIdx.x]) : 0;
  const uint64_t act = ballot(rows > 0);
  int run = rows;
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(run, o, kWave);
    if (lane >= o) run += y;
  }
  if (mine && lane == kWave - 1) {
    s.wave_n[wave] = __popcll(act);
    s.wave_rows[wave] = run;
  }
  __syncthreads();
  if (mine) {
    int n0 = 0, r0 = 0;
    for (int w = 0; w < wave; ++w) {
      n0 += s.wave_n[w];
      r0 += s.wave_rows[w];
    }
    if (rows > 0) s.list[n0 + __popcll(act & lanemask_lt())] = (uint8_t)threadIdx.x;
    s.base[threadIdx.x] = r0 + run - rows;
    if (threadIdx.x == kLdExperts - 1) s.n_active = n0 + __popcll(act);
  }
  __syncthreads();
  for (int q = threadIdx.x; q < T * k; q += THREADS) {
    const int e = s.sel[q], t = q / k;
    if (e < 0 || !((s.mask[e] >> t) & 1)) continue;
    const int r = s.base[e] + __popcll(s.mask[e] & ((1ull << t) - 1));
    s.row_token[r] = (uint8_t)t;
    s.row_gate[r] = s.gate[q];
  }
  __syncthreads();
}

struct LdArgs {
  const void *x, *w_gate, *w_up, *w_down, *sh_gate, *sh_up, *sh_down;
  int64_t H, F, Fs;
  int T, E, k, S, renorm;
  const int32_t* slot;
  const void* w_router;
  const float* bias;
  int bias_mode;
  double* z;
  void* act;
  LdEntry* entries;                              // [E], the first *n_entries hold
  int32_t* n_entries;
  uint8_t* row_token;                            // [T * k]: token of an activation row
  float* part;                                   // [parts][T][H]
  int32_t *topk_idx, *incomplete;
  float* topk_w;
};

// The activation operand of one K block, MT tiles of 16 rows: lane (row r, q)
// needs chunks q and 4 + q of its rows' lines. HALF, at most eight rows: one
// load of 8 rows x 128 bytes and the lane swap, as for weights.
template <int MT, bool HALF>
struct LdRows {
  static constexpr int LOADS = HALF ? 1 : 2 * MT;
  u32x4_t v[LOADS];

  // byte offset of this lane's first chunk in load i, given its row's offset
  template <typename RowOffset>
  static __device__ __forceinline__ void offsets(uint32_t (&off)[HALF ? 1 : MT], int m,
                                                 RowOffset&& row_offset) {
    const int lane = lane_id(), q4 = lane >> 4;
    if constexpr (HALF) {
      off[0] = (lane & 7) < m ? row_offset(lane & 7) + (q4 + ((lane >> 3) & 1) * 4) * 16 : kPastEnd;
    } else {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int row = 16 * i + (lane & 15);
        off[i] = row < m ? row_offset(row) + q4 * 16 : kPastEnd;
      }
    }
  }
  __device__ __forceinline__ void load(rsrc_t rs, const uint32_t (&off)[HALF ? 1 : MT], uint32_t at,
                                       uint32_t row_bytes) {
    const int lane = lane_id(), q4 = lane >> 4;
    if constexpr (HALF) {
      const bool in = at + (q4 + ((lane >> 3) & 1) * 4) * 16 < row_bytes;
      v[0] = buf_load16<false>(rs, in ? off[0] : kPastEnd, at);
    } else {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const bool in = at + hh * 64 + q4 * 16 < row_bytes;
#pragma unroll
        for (int i = 0; i < MT; ++i)
          v[2 * i + hh] = buf_load16<false>(
              rs, in && off[i] != kPastEnd ? off[i] + hh * 64 : kPastEnd, at);
      }
    }
  }
  __device__ __forceinline__ u32x4_t operand(int i, int hh) const {
    if constexpr (!HALF) return v[2 * i + hh];
    u32x4_t o;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o[e] = hh == 0 ? ror8_into(v[0][e], 0u, true) : ror8_into(0u, v[0][e], false);
    return o;
  }
};

// K blocks [b0, b1) in batches of U: all loads of a batch, then its products.
// FENCE (more than 16 tokens) keeps the order: left to the scheduler, loads sink
// between the products of several row tiles and few are in flight (64 tokens of
// the Mixtral shape, down projection 193 us, fenced 175; 24 of the Qwen shape 27.4,
// 24.5); with up to 16 tokens it does as well alone (13 of the DeepSeek shape,
// gate and up 43.9, fenced 46.1).
template <int U, bool FENCE, typename Block, typename Load, typename Use>
__device__ __forceinline__ void ld_stream(int b0, int b1, Load&& load, Use&& use) {
  int b = b0;
  for (; b + U <= b1; b += U) {
    Block k[U];
#pragma unroll
    for (int u = 0; u < U; ++u) load(k[u], b + u);
    if constexpr (FENCE) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) use(k[u]);
  }
  if constexpr (U > 1) {
    if (b < b1) {
      Block k[U - 1];
#pragma unroll
      for (int u = 0; u < U - 1; ++u)
        if (b + u < b1) load(k[u], b + u);
#pragma unroll
      for (int u = 0; u < U - 1; ++u)
        if (b + u < b1) use(k[u]);
    }
  }
}

// ---------------------------------------------------------------- gate and up
// A unit: 16 * NT columns of one expert's gate and up projections for its m
// rows; row i is token tok[i] (token i when NULL), scaled by gate[i]. Each of
// the W waves streams a contiguous part of K of the NT gate and NT up tiles; the
// partial sums are added through LDS in wave order.
template <typename Tv, int MTMAX, int NT, int W>
struct LdUp {
  using LT = LdType<Tv>;
  static constexpr int TILES = 2 * NT, COLS = 16 * NT;
  static constexpr int RC = MTMAX < 2 ? MTMAX : 2;         // row tiles per LDS pass
  using Part = f32x4_t[W][RC][TILES][kWave];

  // K blocks of a batch: as many as leave every instance without a spilled
  // register (at 128 a lane with eight waves, 256 with four)
  static constexpr int unroll(int mt) {
    if (TILES == 2) return mt == 1 ? 3 : mt == 2 ? 2 : 1;
    return mt == 1 ? 2 : 1;
  }

  template <int MT, bool HALF>
  static __device__ __forceinline__ void rows(rsrc_t rs_x, Part& part, int m, const uint8_t* tok,
                                              const float* gate, const Tv* wg, const Tv* wu,
                                              int64_t K, int64_t n0, int64_t N, Tv* out) {
    using X = LdRows<MT, HALF>;
    const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t row_bytes = (uint32_t)(K * sizeof(Tv));
    const int nb = (int)((K + LT::KB - 1) / LT::KB);
    const uint32_t w_chunk = (q4 + ((lane >> 3) & 1) * 4) * 16;   // of the lane's row's line
    const uint32_t w_off = (uint32_t)(lane & 7) * row_bytes + w_chunk;
    const uint32_t w_half = 8 * row_bytes;
    uint32_t x_off[HALF ? 1 : MT];
    X::offsets(x_off, m, [&](int row) { return (uint32_t)(tok ? tok[row] : row) * row_bytes; });
    rsrc_t rs[TILES];
#pragma unroll
    for (int g = 0; g < TILES; ++g) {
      // a tile past N (of the last unit) re-reads the first, not stored
      const int64_t n = n0 + 16 * (g / 2) < N ? n0 + 16 * (g / 2) : n0;
      const int64_t rows = min(N - n, (int64_t)16);
      const Tv* const p = (g % 2 == 0 ? wg : wu) + n * K;
      rs[g] = __builtin_amdgcn_make_buffer_rsrc(const_cast<Tv*>(p), 0, (int)(rows * row_bytes),
                                                0x00027000);
    }
    f32x4_t acc[MT][TILES];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int g = 0; g < TILES; ++g) acc[i][g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    struct Block { u32x4_t w[TILES][2]; X x; };
    ld_stream<unroll(MT), (MTMAX > 1), Block>(
        nb * wave / W, nb * (wave + 1) / W,
        [&](Block& k, int b) {
          const uint32_t at = (uint32_t)b * 128;
          const bool w_in = at + w_chunk < row_bytes;
#pragma unroll
          for (int g = 0; g < TILES; ++g)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
              k.w[g][hh] = buf_load16<true>(rs[g], w_in ? w_off + hh * w_half : kPastEnd, at);
          k.x.load(rs_x, x_off, at, row_bytes);
        },
        [&](const Block& k) {
#pragma unroll
          for (int g = 0; g < TILES; ++g) {
            u32x4_t w0, w1;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              w0[v] = ror8_into(k.w[g][0][v], k.w[g][1][v], true);
              w1[v] = ror8_into(k.w[g][1][v], k.w[g][0][v], false);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              LT::mfma(acc[i][g], k.x.operand(i, 0), w0);
              LT::mfma(acc[i][g], k.x.operand(i, 1), w1);
            }
          }
        });
#pragma unroll
    for (int i0 = 0; i0 < MT; i0 += RC) {
#pragma unroll
      for (int ii = 0; ii < RC; ++ii)
        if (i0 + ii < MT)
#pragma unroll
          for (int g = 0; g < TILES; ++g) part[wave][ii][g][lane] = acc[i0 + ii][g];
      __syncthreads();
      // C layout of the 16x16 MFMA: lane holds column lane % 16, rows 4 * (lane / 16) + q
      for (int gi = wave; gi < (MT - i0 < RC ? MT - i0 : RC) * NT; gi += W) {
        const int i = gi / NT, j = gi % NT;
        f32x4_t g = part[0][i][2 * j][lane], u = part[0][i][2 * j + 1][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) {
          g += part[w][i][2 * j][lane];
          u += part[w][i][2 * j + 1][lane];
        }
        const int64_t col = n0 + 16 * j + r;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int row = 16 * (i0 + i) + 4 * q4 + q;
          // one rounding to the type, of the gated activation: the down
          // projection's operand
          if (row < m && col < N)
            out[row * N + col] = LT::put(LT::act(g[q], u[q]) * (gate ? gate[row] : 1.f));
        }
      }
      __syncthreads();                           // part is rewritten next
    }
  }

  static __device__ __forceinline__ void run(rsrc_t rs_x, Part& part, int m, const uint8_t* tok,
                                             const float* gate, const Tv* wg, const Tv* wu,
                                             int64_t K, int64_t n0, int64_t N, Tv* out) {
    if (m <= 8) rows<1, true>(rs_x, part, m, tok, gate, wg, wu, K, n0, N, out);
    else if (m <= 16) rows<1, false>(rs_x, part, m, tok, gate, wg, wu, K, n0, N, out);
    else if (m <= 32) { if constexpr (MTMAX >= 2) rows<2, false>(rs_x, part, m, tok, gate, wg, wu, K, n0, N, out); }
    else if (m <= 48) { if constexpr (MTMAX >= 4) rows<3, false>(rs_x, part, m, tok, gate, wg, wu, K, n0, N, out); }
    else { if constexpr (MTMAX >= 4) rows<4, false>(rs_x, part, m, tok, gate, wg, wu, K, n0, N, out); }
  }
};

template <typename Tv>
__device__ __forceinline__ rsrc_t ld_x(const LdArgs& a) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(a.x), 0,
                                           (int)(a.T * (uint32_t)(a.H * sizeof(Tv))), 0x00027000);
}

// The logits: a block one expert, a token a wave.
constexpr int kLogitWaves = 4;

template <typename Tv>
__global__ void __launch_bounds__(64 * kLogitWaves)
ld_first_kernel(LdArgs a) {
  const int t = blockIdx.x / a.E * kLogitWaves + threadIdx.x / kWave;
  if (t < a.T)
    ld_logit(static_cast<const Tv*>(a.x), static_cast<const Tv*>(a.w_router), t,
             (int)(blockIdx.x % a.E), a.H, a.E, a.bias, a.bias_mode, a.z);
}

// What the call returns of the routes and the launch after reads, by the whole block.
template <int TOK>
__device__ __forceinline__ void ld_write_routes(const LdArgs& a, const LdRoutes<TOK>& rt) {
  const int threads = blockDim.x;
  for (int q = threadIdx.x; q < a.T * a.k; q += threads) {
    a.topk_idx[q] = rt.sel[q];
    a.topk_w[q] = rt.gate[q];
    a.row_token[q] = rt.row_token[q];
  }
  for (int t = threadIdx.x; a.incomplete && t < a.T; t += threads) {
    int miss = 0;
    for (int j = 0; j < a.k; ++j) {
      const int e = rt.sel[t * a.k + j];
      miss |= e >= 0 && !((rt.mask[e] >> t) & 1);
    }
    a.incomplete[t] = miss;
  }
  for (int q = threadIdx.x; q < rt.n_active; q += threads) {
    const int e = rt.list[q];
    a.entries[q] = LdEntry{rt.slot[e], rt.base[e], (int)__popcll(rt.mask[e])};
  }
  if (threadIdx.x == 0) *a.n_entries = rt.n_active;
}

// The first blocks stream the shared experts' units, which need no route, while the
// others decide the routes and then stream the units of the active experts (logits,
// gate and up of a Qwen-shaped token 23.4 us, with the shared units beside the
// logits 30; of 64 75, 91).
template <typename Tv, int MTMAX, int NT, int W>
__global__ void __launch_bounds__(64 * W, W / 2)
ld_up_kernel(LdArgs a, int shared_blocks) {
  using Up = LdUp<Tv, MTMAX, NT, W>;
  constexpr int THREADS = 64 * W;
  __shared__ LdRoutes<16 * MTMAX> rt;
  __shared__ typename Up::Part part;
  const int sb = blockIdx.x, rb = sb - shared_blocks;
  if (rb < 0) {
    Tv* const act = static_cast<Tv*>(a.act) + (int64_t)a.T * a.k * a.F;
    const int units = (int)((a.Fs + Up::COLS - 1) / Up::COLS);
    for (int unit = sb; unit < units; unit += shared_blocks)
      Up::run(ld_x<Tv>(a), part, a.T, nullptr, nullptr, static_cast<const Tv*>(a.sh_gate),
              static_cast<const Tv*>(a.sh_up), a.H, (int64_t)unit * Up::COLS, a.Fs, act);
    return;
  }
  ld_routes<16 * MTMAX, THREADS>(a.z, a.T, a.E, a.k, a.renorm, a.slot, a.S, rt);
  if (rb == 0) ld_write_routes(a, rt);
  const int ncb = (int)((a.F + Up::COLS - 1) / Up::COLS);
  const int units = __builtin_amdgcn_readfirstlane(rt.n_active) * ncb;
  const int step = gridDim.x - shared_blocks;
  for (int unit = rb; unit < units; unit += step) {
    const int e = __builtin_amdgcn_readfirstlane(rt.list[unit / ncb]);
    const int base = __builtin_amdgcn_readfirstlane(rt.base[e]);
    const int m = __builtin_amdgcn_readfirstlane(__popcll(rt.mask[e]));
    const int64_t sl = __builtin_amdgcn_readfirstlane(rt.slot[e]);
    Up::run(ld_x<Tv>(a), part, m, rt.row_token + base, rt.row_gate + base,
            static_cast<const Tv*>(a.w_gate) + sl * a.F * a.H,
            static_cast<const Tv*>(a.w_up) + sl * a.F * a.H, a.H,
            (int64_t)(unit % ncb) * Up::COLS, a.F,
            static_cast<Tv*>(a.act) + (int64_t)base * a.F);
  }
}

// ---------------------------------------------------------------- down
// A block owns COLS columns of y. The K blocks of all active experts and the
// shared ones form one sequence, cut into contiguous ranges of the waves; a wave
// keeps a sum for every token in LDS, to which it adds an expert's rows when it
// leaves the expert, and the waves' sums are added in wave order.
// COLS 16 or 8, sixteen waves: one block a compute unit has enough loads in
// flight, and it sees the whole sequence, so the sum is y. COLS 64, four waves:
// four weight tiles beside each activation load; the sequence is cut over blocks
// too, whose float32 sums ld_join_kernel adds up.
constexpr int ld_down_waves(int cols) { return cols == 64 ? 4 : 16; }

template <typename Tv, int MTMAX, int COLS>
struct LdDown {
  using LT = LdType<Tv>;
  static constexpr int NT = COLS / 16 > 1 ? COLS / 16 : 1;   // weight tiles
  static constexpr int WL = COLS == 8 ? 1 : 2;   // loads of a tile per K block
  static constexpr int WAVES = ld_down_waves(COLS);
  using Sum = float[16 * MTMAX][16 * NT];

  // K blocks of a batch: as many as leave every instance without a spilled
  // register (at 128 a lane with sixteen waves, 256 with four)
  static constexpr int unroll(int mt, bool half) {
    if (COLS == 64) return half ? 3 : 2;
    if (COLS == 8) return half ? 8 : mt == 1 ? 5 : mt == 2 ? 3 : 2;
    return half ? 5 : mt == 1 ? 4 : mt == 2 ? 3 : 2;
  }

  // sum[token][column] += rows' products over K blocks [b0, b1) of an expert:
  // weight rows at w, activation rows from byte `first` on
  template <int MT, bool HALF>
  static __device__ __forceinline__ void rows(Sum& sum, rsrc_t rs_a, const Tv* w, int64_t K,
                                              int64_t n_rows, uint32_t first, int m,
                                              const uint8_t* tok, int b0, int b1) {
    using X = LdRows<MT, HALF>;
    const int lane = lane_id(), r = lane & 15, q4 = lane >> 4;
    const uint32_t row_bytes = (uint32_t)(K * sizeof(Tv));
    const uint32_t w_chunk = (q4 + ((lane >> 3) & 1) * 4) * 16;
    const uint32_t w_off = (uint32_t)(lane & 7) * row_bytes + w_chunk;
    rsrc_t rs[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      // a tile past y's columns re-reads the first, not stored
      const int64_t n = 16 * j < n_rows ? 16 * j : 0;
      rs[j] = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<Tv*>(w + n * K), 0,
          (int)((uint32_t)min(n_rows - n, (int64_t)(8 * WL)) * row_bytes), 0x00027000);
    }
    uint32_t x_off[HALF ? 1 : MT];
    X::offsets(x_off, m, [&](int row) { return first + (uint32_t)row * row_bytes; });
    f32x4_t acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    struct Block { u32x4_t w[NT][WL]; X x; };
    ld_stream<unroll(MT, HALF), (MTMAX > 1), Block>(
        b0, b1,
        [&](Block& k, int b) {
          const uint32_t at = (uint32_t)b * 128;
          const bool w_in = at + w_chunk < row_bytes;
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int hh = 0; hh < WL; ++hh)
              k.w[j][hh] = buf_load16<true>(rs[j], w_in ? w_off + hh * 8 * row_bytes : kPastEnd, at);
          k.x.load(rs_a, x_off, at, row_bytes);
        },
        [&](const Block& k) {
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            u32x4_t w0, w1;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              // eight columns: the tile's other eight are zeros
              const uint32_t other = WL == 2 ? k.w[j][WL - 1][v] : 0u;
              w0[v] = ror8_into(k.w[j][0][v], other, true);
              w1[v] = ror8_into(other, k.w[j][0][v], false);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              LT::mfma(acc[i][j], k.x.operand(i, 0), w0);
              LT::mfma(acc[i][j], k.x.operand(i, 1), w1);
            }
          }
        });
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = 16 * i + 4 * q4 + q;
        if (row >= m) continue;
        const int t = tok ? tok[row] : row;
#pragma unroll
        for (int j = 0; j < NT; ++j) sum[t][16 * j + r] += acc[i][j][q];
      }
    __builtin_amdgcn_wave_barrier();             // another lane may add to the same next
    asm volatile("" ::: "memory");
  }
};

template <typename Tv, int MTMAX, int COLS>
__global__ void __launch_bounds__(64 * ld_down_waves(COLS))
ld_down_kernel(LdArgs a, int accumulate, Tv* __restrict__ y) {
  using Down = LdDown<Tv, MTMAX, COLS>;
  using LT = LdType<Tv>;
  constexpr int WAVES = Down::WAVES, THREADS = 64 * WAVES, W16 = 16 * Down::NT;
  __shared__ LdEntry ent[kLdExperts];
  __shared__ uint8_t row_token[16 * MTMAX * kLdMaxK];
  __shared__ typename Down::Sum sum[WAVES];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // everything the launch before left, at once (entries past the last are not used)
  const int n_ent = __builtin_amdgcn_readfirstlane(*a.n_entries);
  for (int q = threadIdx.x; q < a.E; q += THREADS) ent[q] = a.entries[q];
  for (int q = threadIdx.x; q < a.T * a.k; q += THREADS) row_token[q] = a.row_token[q];
  for (int q = lane; q < 16 * MTMAX * W16; q += kWave) (&sum[wave][0][0])[q] = 0.f;
  __syncthreads();
  const int64_t n0 = (int64_t)blockIdx.x * COLS;
  const int64_t n_rows = min(a.H - n0, (int64_t)COLS);
  const int nb = (int)((a.F + LT::KB - 1) / LT::KB), nbs = (int)((a.Fs + LT::KB - 1) / LT::KB);
  const int64_t total = (int64_t)n_ent * nb + nbs;
  const int64_t part = (int64_t)blockIdx.y * WAVES + wave, parts = (int64_t)gridDim.y * WAVES;
  const int64_t lo = total * part / parts, hi = total * (part + 1) / parts;
  const uint32_t act_bytes = (uint32_t)(((int64_t)a.T * a.k * a.F + a.T * a.Fs) * sizeof(Tv));
  const rsrc_t rs_a = __builtin_amdgcn_make_buffer_rsrc(a.act, 0, (int)act_bytes, 0x00027000);
  // the place in the sequence: entry (n_ent: shared) and K block in it
  int en = (int)min(lo / nb, (int64_t)n_ent);
  int kb = (int)(lo - (int64_t)en * nb);
  for (int64_t g = lo; g < hi;) {
    const bool sh = en >= n_ent;
    const int64_t K = sh ? a.Fs : a.F;
    const Tv* w = static_cast<const Tv*>(a.sh_down) + n0 * K;
    uint32_t first = (uint32_t)((int64_t)a.T * a.k * a.F * sizeof(Tv));
    int m = a.T;
    const uint8_t* tok = nullptr;
    if (!sh) {
      const int64_t sl = __builtin_amdgcn_readfirstlane(ent[en].slot);
      const int base = __builtin_amdgcn_readfirstlane(ent[en].base);
      m = __builtin_amdgcn_readfirstlane(ent[en].rows);
      first = (uint32_t)base * (uint32_t)(K * sizeof(Tv));
      tok = row_token + base;
      w = static_cast<const Tv*>(a.w_down) + (sl * a.H + n0) * K;
    }
    const int b1 = (int)min((int64_t)(sh ? nbs : nb), kb + (hi - g));
    typename Down::Sum& s = sum[wave];
    if (m <= 8) Down::template rows<1, true>(s, rs_a, w, K, n_rows, first, m, tok, kb, b1);
    else if (m <= 16) Down::template rows<1, false>(s, rs_a, w, K, n_rows, first, m, tok, kb, b1);
    else if (m <= 32) { if constexpr (MTMAX >= 2) Down::template rows<2, false>(s, rs_a, w, K, n_rows, first, m, tok, kb, b1); }
    else if (m <= 48) { if constexpr (MTMAX >= 4) Down::template rows<3, false>(s, rs_a, w, K, n_rows, first, m, tok, kb, b1); }
    else { if constexpr (MTMAX >= 4) Down::template rows<4, false>(s, rs_a, w, K, n_rows, first, m, tok, kb, b1); }
    g += b1 - kb;
    ++en;
    kb = 0;
  }
  __syncthreads();
  for (int q = threadIdx.x; q < a.T * W16; q += THREADS) {
    const int t = q / W16, c = q % W16;
    if (c >= n_rows) continue;
    float v = sum[0][t][c];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += sum[w][t][c];
    if constexpr (COLS == 64) {
      a.part[((int64_t)blockIdx.y * a.T + t) * a.H + n0 + c] = v;
    } else {
      Tv* const o = y + t * a.H + n0 + c;
      *o = LT::put(accumulate ? v + LT::get(*o) : v);
    }
  }
}

// y = (y +) the parts' sums, in part order; four columns a thread (H is a
// multiple of four).
template <typename Tv>
__global__ void __launch_bounds__(256)
ld_join_kernel(LdArgs a, int parts, int accumulate, Tv* __restrict__ y) {
  using LT = LdType<Tv>;
  const int64_t n = (int64_t)a.T * a.H, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= n) return;
  f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.part + at);
  for (int p = 1; p < parts; ++p) v += *reinterpret_cast<const f32x4_t*>(a.part + p * n + at);
#pragma unroll
  for (int e = 0; e < 4; ++e) y[at + e] = LT::put(accumulate ? v[e] + LT::get(y[at + e]) : v[e]);
}

// Experts that can be active.
int64_t ld_experts(const LdArgs& a) {
  return std::min<int64_t>((int64_t)a.T * a.k, std::min(a.E, a.S));
}

template <typename Tv, int MTMAX, int NT, int W>
int ld_up(const LdArgs& a, hipStream_t st) {
  const int64_t units = ld_experts(a) * ceil_div(a.F, 16 * NT), most = 2 * device_cu_count();
  const int shared = (int)std::min<int64_t>(ceil_div(a.Fs, 16 * NT), most);
  const unsigned grid = (unsigned)(shared + std::min<int64_t>(units, most));
  ld_up_kernel<Tv, MTMAX, NT, W><<<dim3(grid), dim3(64 * W), 0, st>>>(a, shared);
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv, int MTMAX>
int ld_launch(const LdArgs& a, int accumulate, Tv* y, hipStream_t st) {
  // gate and up: units of 32 columns and four waves when they give every compute
  // unit two (32 Mixtral-shaped tokens 282 us, by narrow units 319; 13
  // DeepSeek-shaped 44, 53), else of 16 columns and eight waves, which have all of
  // K in flight (the four experts of a Qwen-shaped token 16.4 us, by wide units 18.0)
  const int64_t cus = device_cu_count(), experts = ld_experts(a);
  ld_first_kernel<Tv><<<dim3((unsigned)(a.E * ceil_div(a.T, kLogitWaves))),
                        dim3(64 * kLogitWaves), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  int rc;
  if constexpr (MTMAX == 4) {                    // four row tiles need the registers of wide units
    rc = ld_up<Tv, MTMAX, 2, 4>(a, st);
  } else {
    rc = experts * ceil_div(a.F, 32) >= 2 * cus ? ld_up<Tv, MTMAX, 2, 4>(a, st)
                                                : ld_up<Tv, MTMAX, 1, 8>(a, st);
  }
  if (rc != MOE_OK) return rc;
  if constexpr (MTMAX > 1) {
    const int parts = ld_parts(a.T, a.H);
    ld_down_kernel<Tv, MTMAX, 64>
        <<<dim3((unsigned)ceil_div(a.H, 64), (unsigned)parts), dim3(64 * ld_down_waves(64)), 0, st>>>(
            a, accumulate, y);
    MOE_CHECK_LAUNCH();
    ld_join_kernel<Tv><<<dim3((unsigned)ceil_div(a.T * a.H, 1024)), dim3(256), 0, st>>>(
        a, parts, accumulate, y);
  } else if (ceil_div(a.H, 16) < cus) {
    // eight columns a block where sixteen leave compute units idle (a Qwen-shaped
    // token 11.6 us, 16.4)
    ld_down_kernel<Tv, MTMAX, 8>
        <<<dim3((unsigned)ceil_div(a.H, 8)), dim3(64 * ld_down_waves(8)), 0, st>>>(a, accumulate, y);
  } else {
    ld_down_kernel<Tv, MTMAX, 16>
        <<<dim3((unsigned)ceil_div(a.H, 16)), dim3(64 * ld_down_waves(16)), 0, st>>>(a, accumulate, y);
  }
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv>
int ld_run(const LdArgs& a, int accumulate, void* y, hipStream_t st) {
  Tv* const out = static_cast<Tv*>(y);
  if (a.T <= 16) return ld_launch<Tv, 1>(a, accumulate, out, st);
  if (a.T <= 32) return ld_launch<Tv, 2>(a, accumulate, out, st);
  return ld_launch<Tv, 4>(a, accumulate, out, st);
}

bool ld_ok(int64_t T, int64_t H, int64_t F, int32_t E, int32_t k, int64_t Fs, int32_t dtype) {
  return T >= 1 && H >= 1 && F >= 1 && E >= 1 && E <= kLdExperts && k >= 1 && k <= E && Fs >= 0 &&
         valid_dtype(dtype);
}
bool ld_supported(int64_t T, int64_t H, int64_t F, int32_t E, int32_t k, int64_t Fs,
                  int32_t dtype) {
  const int64_t ve = dtype == MOE_BF16 ? 8 : 4;
  // 32-bit byte offsets within 16 weight rows, all tokens and the activations
  const int64_t lim = (int64_t)1 << 24;
  if (T > kLdTokens || k > kLdMaxK || H % ve || F % ve || Fs % ve) return false;
  if (H > lim / 4 || F > lim || Fs > lim) return false;
  return act_rows_bytes(T, k, F, Fs, 16 / ve) < (int64_t)kPastEnd;
}

}  // namespace
}  // namespace moe

extern "C" size_t moe_layer_decode_workspace(int64_t T, int64_t H, int64_t F, int32_t E, int32_t k,
                                             int64_t Fs, int32_t dtype) {
  if (!moe::ld_ok(T, H, F, E, k, Fs, dtype) || !moe::ld_supported(T, H, F, E, k, Fs, dtype))
    return 0;
  return moe::ld_layout(T, H, F, E, k, Fs, dtype).total;
}

extern "C" int moe_layer_decode(const void* x, int32_t dtype, int64_t T, int64_t H,
                                const void* w_router, int32_t E, int32_t k, const float* bias,
                                int32_t bias_mode, int32_t renormalize, const void* w_gate,
                                const void* w_up, const void* w_down, int32_t S, int64_t F,
                                const int32_t* slot_of_expert, const void* shared_gate,
                                const void* shared_up, const void* shared_down, int64_t Fs,
                                int32_t accumulate, void* y, int32_t* topk_idx, float* topk_w,
                                int32_t* incomplete, void* workspace, size_t ws_bytes,
                                void* stream) {
  using namespace moe;
  MOE_CHECK_ARG(x && w_router && w_gate && w_up && w_down && y && topk_idx && topk_w);
  MOE_CHECK_ARG(ld_ok(T, H, F, E, k, Fs, dtype));
  MOE_CHECK_ARG(S >= 1 && (slot_of_expert || S >= E));
  MOE_CHECK_ARG(bias_mode >= 0 && bias_mode <= 2 && (bias_mode == 0) == (bias == nullptr));
  MOE_CHECK_ARG((renormalize == 0 || renormalize == 1) && (accumulate == 0 || accumulate == 1));
  MOE_CHECK_ARG(Fs == 0 ? !shared_gate && !shared_up && !shared_down
                        : shared_gate && shared_up && shared_down);
  if (!ld_supported(T, H, F, E, k, Fs, dtype)) return MOE_ERR_UNSUPPORTED;
  uintptr_t bits = 0;
  for (const void* p : {x, w_router, w_gate, w_up, w_down, shared_gate, shared_up, shared_down,
                        static_cast<const void*>(y)})
    bits |= reinterpret_cast<uintptr_t>(p);
  if (bits & 15) return MOE_ERR_UNSUPPORTED;     // 16-byte loads
  const LdLayout lay = ld_layout(T, H, F, E, k, Fs, dtype);
  if (!workspace || ws_bytes < lay.total || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return MOE_ERR_WORKSPACE;
  char* const ws = static_cast<char*>(workspace);
  LdArgs a{};
  a.x = x;
  a.w_gate = w_gate;
  a.w_up = w_up;
  a.w_down = w_down;
  a.sh_gate = shared_gate;
  a.sh_up = shared_up;
  a.sh_down = shared_down;
  a.H = H;
  a.F = F;
  a.Fs = Fs;
  a.T = (int)T;
  a.E = E;
  a.k = k;
  a.S = S;
  a.renorm = renormalize;
  a.slot = slot_of_expert;
  a.w_router = w_router;
  a.bias = bias;
  a.bias_mode = bias_mode;
  a.z = reinterpret_cast<double*>(ws + lay.z);
  a.act = ws + lay.act;
  a.entries = reinterpret_cast<LdEntry*>(ws + lay.entries);
  a.n_entries = reinterpret_cast<int32_t*>(ws + lay.meta);
  a.row_token = reinterpret_cast<uint8_t*>(ws + lay.tokens);
  a.part = reinterpret_cast<float*>(ws + lay.part);
  a.topk_idx = topk_idx;
  a.topk_w = topk_w;
  a.incomplete = incomplete;
  hipStream_t st = as_stream(stream);
  return dtype == MOE_BF16 ? ld_run<uint16_t>(a, accumulate, y, st)
                           : ld_run<float>(a, accumulate, y, st);
}
