// moe_layer_decode: a whole MoE layer (router, top-k gates, SwiGLU experts over
// the resident slots, shared experts, weighted sum) for at most 64 tokens.
//
// So few tokens leave the layer bound by reading the weights of the experts
// they reach once (HBM); the rest is launches and latencies, so there are three
// of the former and no permuted copies:
//   ld_logits_kernel  the router's logits in float64, spread over the chip
//   ld_up_kernel      every block decides the routes of all tokens for itself
//                     (a microsecond; it needs no other block), then the blocks
//                     stream gate and up rows and write
//                       a[t, :] = gate_t * silu(x_t . Wg^T) * (x_t . Wu^T)
//   ld_down_kernel    y[t, n] = sum over the experts of t of a . Wd[n, :]: the
//                     gates are in a, so the sums of all experts of a column
//                     tile run on in the same accumulators
// No block waits for another except for the join of the last launch's K parts,
// which the last block of a column tile to arrive does, in a fixed order.
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
constexpr int kLdThreads = 256, kLdWaves = kLdThreads / kWave;
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

// An expert that tokens reached and that is resident: `rows` of the activation
// from `base` on belong to the tokens of `mask`, ascending.
struct LdEntry {
  uint64_t mask;
  int32_t slot, base;
};

struct LdLayout {
  size_t z, meta, entries, act, part, count, total;
  int parts;                                     // K parts of the down projection
  int64_t col_tiles;                             // its column tiles
};

constexpr int kDownTiles = 1;                    // 16-column tiles of a down block

int64_t act_rows_bytes(int64_t T, int32_t k, int64_t F, int64_t Fs, size_t elt) {
  return (int64_t)((size_t)T * k * F * elt + (size_t)T * Fs * elt);
}

LdLayout ld_layout(int64_t T, int64_t H, int64_t F, int32_t E, int32_t k, int64_t Fs,
                   int32_t dtype) {
  const size_t elt = dtype == MOE_BF16 ? 2 : 4;
  LdLayout s{};
  s.col_tiles = ceil_div(H, 16 * kDownTiles);
  // enough blocks for two a compute unit, K parts of a wave not below four K
  // blocks of a single expert
  const int64_t kb = dtype == MOE_BF16 ? 64 : 32;
  const int64_t blocks = ceil_div(F, kb) * std::min<int64_t>(k, E) + ceil_div(Fs, kb);
  int64_t p = ceil_div(512, s.col_tiles);
  p = std::min(p, std::max<int64_t>(1, blocks / (4 * kLdWaves)));
  s.parts = (int)std::min<int64_t>(std::max<int64_t>(p, 1), 16);
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = align_up(o + bytes, 256);
    return at;
  };
  s.z = take((size_t)T * E * 8);
  s.meta = take(4);
  s.entries = take((size_t)E * sizeof(LdEntry));
  s.act = take((size_t)act_rows_bytes(T, k, F, Fs, elt));
  s.part = take(s.parts > 1 ? (size_t)s.parts * s.col_tiles * 16 * kDownTiles * align_up(T, 16) * 4 : 0);
  s.count = take((size_t)s.col_tiles * 4);
  s.total = o;
  return s;
}

// ---------------------------------------------------------------- logits
// z[t, e] in float64 (bf16 products are exact in it): one wave a (token,
// expert), four tokens a block. Block 0 clears the counters of the last launch.
template <typename Tv>
__global__ void __launch_bounds__(kLdThreads)
ld_logits_kernel(const Tv* __restrict__ x, const Tv* __restrict__ wr, int T, int64_t H, int E,
                 const float* __restrict__ bias, int bias_mode, double* __restrict__ z,
                 int32_t* __restrict__ count, int64_t n_count) {
  constexpr int VE = 16 / sizeof(Tv);
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int e = blockIdx.x;
  const int t = blockIdx.y * kLdWaves + wave;
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int64_t q = threadIdx.x; q < n_count; q += kLdThreads) count[q] = 0;
  if (t >= T) return;
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
// What a block keeps of the routes of all tokens.
struct LdRoutes {
  uint64_t mask[kLdExperts];                     // tokens that chose a resident expert
  float gate[kLdTokens * kLdMaxK];               // by token and choice
  float row_gate[kLdTokens * kLdMaxK];           // by activation row
  int16_t sel[kLdTokens * kLdMaxK];              // expert of a choice, -1: none
  int32_t base[kLdExperts];
  uint8_t row_token[kLdTokens * kLdMaxK];
  uint8_t list[kLdExperts];                      // active experts, ascending
  int32_t wave_n[kLdWaves], wave_rows[kLdWaves];
  int32_t n_active;
};

// Top-k (larger logit, then lower expert; a NaN is never chosen) and gates of
// token t by the 16 lanes of a row; lane gl holds the logits of experts
// gl + 16 r. k rounds of row arg-max; the gates are float32 exponentials of
// float64 differences.
template <int EPL>
__device__ __forceinline__ void ld_decide(const double* __restrict__ z, bool live, int t, int E,
                                          int k, int renorm, int gl, LdRoutes& s) {
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
  float total = 0.f, chosen = 0.f;
  if (!renorm) {
#pragma unroll
    for (int r = 0; r < EPL; ++r)
      if (live && gl + kRowLanes * r < E) total += expf((float)(v[r] - m));
    total += dpp<0xB1>(total);
    total += dpp<0x4E>(total);
    total += dpp<0x141>(total);
    total += dpp<0x140>(total);
  }
  for (int j = 0; j < k; ++j) {
    double bv = 0.0;
    int be = -1;
#pragma unroll
    for (int r = 0; r < EPL; ++r)
      if (((free >> r) & 1) && (be < 0 || v[r] > bv)) {
        bv = v[r];
        be = gl + kRowLanes * r;
      }
    row_argmax(bv, be);
    const float g = be >= 0 ? expf((float)(bv - m)) : 0.f;
    chosen += g;
    if (be >= 0 && (be & (kRowLanes - 1)) == gl) free &= ~(1u << (be / kRowLanes));
    if (live && gl == 0) {
      s.sel[t * k + j] = (int16_t)be;
      s.gate[t * k + j] = g;
    }
  }
  // each token's gates were written by lane 0 of the row, which divides them too
  if (live && gl == 0) {
    const float den = renorm ? chosen : total;
    for (int j = 0; j < k; ++j) s.gate[t * k + j] = s.gate[t * k + j] / den;
  }
}

// The routes of all tokens, by the whole block; ends with a barrier.
__device__ __forceinline__ void ld_routes(const double* __restrict__ z, int T, int E, int k,
                                          int renorm, const int32_t* __restrict__ slot, int S,
                                          LdRoutes& s) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int gl = lane % kRowLanes, grp = lane / kRowLanes;
  for (int e = threadIdx.x; e < kLdExperts; e += kLdThreads) s.mask[e] = 0;
  for (int t0 = 0; t0 < T; t0 += kLdThreads / kRowLanes) {
    const int t = t0 + wave * (kWave / kRowLanes) + grp;
    const bool live = t < T;
    if (E <= 16) ld_decide<1>(z, live, live ? t : 0, E, k, renorm, gl, s);
    else if (E <= 64) ld_decide<4>(z, live, live ? t : 0, E, k, renorm, gl, s);
    else ld_decide<16>(z, live, live ? t : 0, E, k, renorm, gl, s);
  }
  __syncthreads();
  for (int q = threadIdx.x; q < T * k; q += kLdThreads) {
    const int e = s.sel[q];
    if (e < 0) continue;
    const int sl = slot ? slot[e] : e;
    if (sl >= 0 && sl < S)
      atomicOr(reinterpret_cast<unsigned long long*>(&s.mask[e]), 1ull << (q / k));
  }
  __syncthreads();
  // one thread per expert: its place in the list and its first activation row
  static_assert(kLdThreads >= kLdExperts, "one thread per expert");
  const int rows = __popcll(s.mask[threadIdx.x]);
  const uint64_t act = ballot(rows > 0);
  int run = rows;
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(run, o, kWave);
    if (lane >= o) run += y;
  }
  if (lane == kWave - 1) {
    s.wave_n[wave] = __popcll(act);
    s.wave_rows[wave] = run;
  }
  __syncthreads();
  int n0 = 0, r0 = 0;
  for (int w = 0; w < wave; ++w) {
    n0 += s.wave_n[w];
    r0 += s.wave_rows[w];
  }
  if (rows > 0) s.list[n0 + __popcll(act & lanemask_lt())] = (uint8_t)threadIdx.x;
  s.base[threadIdx.x] = r0 + run - rows;
  if (threadIdx.x == kLdThreads - 1) s.n_active = n0 + __popcll(act);
  __syncthreads();
  for (int q = threadIdx.x; q < T * k; q += kLdThreads) {
    const int e = s.sel[q], t = q / k;
    if (e < 0 || !((s.mask[e] >> t) & 1)) continue;
    const int r = s.base[e] + __popcll(s.mask[e] & ((1ull << t) - 1));
    s.row_token[r] = (uint8_t)t;
    s.row_gate[r] = s.gate[q];
  }
  __syncthreads();
}

// K blocks of a wave loaded per batch, so that some 16 weight loads are in
// flight beside the activations
template <int MT, int TILES>
constexpr int ld_unroll() {
  return (MT == 1 ? 8 : MT == 2 ? 4 : 2) / TILES > 0 ? (MT == 1 ? 8 : MT == 2 ? 4 : 2) / TILES : 1;
}

struct LdArgs {
  const void *x, *w_gate, *w_up, *w_down, *sh_gate, *sh_up, *sh_down;
  int64_t H, F, Fs;
  int T, E, k, S, renorm;
  const int32_t* slot;
  const double* z;
  void* act;
  LdEntry* entries;
  int32_t* n_entries;
  int32_t *topk_idx, *incomplete;
  float* topk_w;
};

// ---------------------------------------------------------------- gate and up
// Units: 16 * NT columns of the shared experts, then of each active expert. A
// wave streams a quarter of K of the unit's NT gate and NT up tiles; the four
// partial sums are added through LDS in order.
template <typename Tv, int MTMAX, int NT>
__global__ void __launch_bounds__(kLdThreads, 2)
ld_up_kernel(LdArgs a) {
  using LT = LdType<Tv>;
  constexpr int TILES = 2 * NT, COLS = 16 * NT;
  __shared__ LdRoutes rt;
  __shared__ f32x4_t part[kLdWaves][MTMAX][TILES][kWave];
  ld_routes(a.z, a.T, a.E, a.k, a.renorm, a.slot, a.S, rt);
  if (blockIdx.x == 0) {
    for (int q = threadIdx.x; q < a.T * a.k; q += kLdThreads) {
      a.topk_idx[q] = rt.sel[q];
      a.topk_w[q] = rt.gate[q];
    }
    for (int t = threadIdx.x; a.incomplete && t < a.T; t += kLdThreads) {
      int miss = 0;
      for (int j = 0; j < a.k; ++j) {
        const int e = rt.sel[t * a.k + j];
        miss |= e >= 0 && !((rt.mask[e] >> t) & 1);
      }
      a.incomplete[t] = miss;
    }
    for (int q = threadIdx.x; q < rt.n_active; q += kLdThreads) {
      const int e = rt.list[q];
      a.entries[q] = LdEntry{rt.mask[e], a.slot ? a.slot[e] : e, rt.base[e]};
    }
    if (threadIdx.x == 0) *a.n_entries = rt.n_active;
  }
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane & 15, q4 = lane >> 4;
  const int64_t K = a.H;
  const uint32_t row_bytes = (uint32_t)(K * sizeof(Tv));
  const int nb = (int)((K + LT::KB - 1) / LT::KB);
  const int b_lo = nb * wave / kLdWaves, b_hi = nb * (wave + 1) / kLdWaves;
  const uint32_t w_chunk = (q4 + ((lane >> 3) & 1) * 4) * 16;   // of the lane's row's line
  const uint32_t w_off = (uint32_t)(lane & 7) * row_bytes + w_chunk;
  const uint32_t w_half = 8 * row_bytes;
  const rsrc_t rs_x = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(a.x), 0,
                                                        (int)(a.T * row_bytes), 0x00027000);
  // rows m of the unit: token of row i is tok[i] (all tokens when NULL)
  auto run_unit = [&](auto mt_c, int m, const uint8_t* tok, const float* gate, const Tv* wg,
                      const Tv* wu, int64_t n0, int64_t N, Tv* out) {
    constexpr int MT = decltype(mt_c)::value;
    constexpr int U = ld_unroll<MT, TILES>();
    uint32_t a_off[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int row = 16 * i + r;
      a_off[i] = row < m ? (uint32_t)(tok ? tok[row] : row) * row_bytes + q4 * 16 : kPastEnd;
    }
    rsrc_t rs[TILES];
#pragma unroll
    for (int g = 0; g < TILES; ++g) {
      // a tile past N (the last unit's second) re-reads the first, not stored
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
    for (int b0 = b_lo; b0 < b_hi; b0 += U) {
      u32x4_t w[U][TILES][2], x[U][MT][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (b0 + u >= b_hi) break;
        const uint32_t at = (uint32_t)(b0 + u) * 128;
        const uint32_t wo = at + w_chunk < row_bytes ? w_off : kPastEnd;
#pragma unroll
        for (int g = 0; g < TILES; ++g)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh)
            w[u][g][hh] = buf_load16<true>(rs[g], wo == kPastEnd ? kPastEnd : wo + hh * w_half, at);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const bool in = at + hh * 64 + q4 * 16 < row_bytes;
#pragma unroll
          for (int i = 0; i < MT; ++i)
            x[u][i][hh] = buf_load16<false>(rs_x, in && a_off[i] != kPastEnd ? a_off[i] + hh * 64 : kPastEnd, at);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (b0 + u >= b_hi) break;
#pragma unroll
        for (int g = 0; g < TILES; ++g) {
          u32x4_t w0, w1;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            w0[v] = ror8_into(w[u][g][0][v], w[u][g][1][v], true);
            w1[v] = ror8_into(w[u][g][1][v], w[u][g][0][v], false);
          }
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            LT::mfma(acc[i][g], x[u][i][0], w0);
            LT::mfma(acc[i][g], x[u][i][1], w1);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int g = 0; g < TILES; ++g) part[wave][i][g][lane] = acc[i][g];
    __syncthreads();
    // C layout of the 16x16 MFMA: lane holds column lane % 16, rows 4 * (lane / 16) + q
    for (int gi = wave; gi < MT * NT; gi += kLdWaves) {
      const int i = gi / NT, j = gi % NT;
      f32x4_t g = part[0][i][2 * j][lane], u = part[0][i][2 * j + 1][lane];
#pragma unroll
      for (int w = 1; w < kLdWaves; ++w) {
        g += part[w][i][2 * j][lane];
        u += part[w][i][2 * j + 1][lane];
      }
      const int64_t col = n0 + 16 * j + r;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = 16 * i + 4 * q4 + q;
        // one rounding to the type, of the gated activation: the down
        // projection's operand
        if (row < m && col < N)
          out[row * N + col] = LT::put(LT::act(g[q], u[q]) * (gate ? gate[row] : 1.f));
      }
    }
    __syncthreads();                             // part is rewritten next
  };
  auto dispatch = [&](int m, const uint8_t* tok, const float* gate, const Tv* wg, const Tv* wu,
                      int64_t n0, int64_t N, Tv* out) {
    if (m <= 16) run_unit(std::integral_constant<int, 1>{}, m, tok, gate, wg, wu, n0, N, out);
    else if (m <= 32) { if constexpr (MTMAX >= 2) run_unit(std::integral_constant<int, 2>{}, m, tok, gate, wg, wu, n0, N, out); }
    else if (m <= 48) { if constexpr (MTMAX >= 4) run_unit(std::integral_constant<int, 3>{}, m, tok, gate, wg, wu, n0, N, out); }
    else { if constexpr (MTMAX >= 4) run_unit(std::integral_constant<int, 4>{}, m, tok, gate, wg, wu, n0, N, out); }
  };
  const int ncb_s = (int)((a.Fs + COLS - 1) / COLS), ncb = (int)((a.F + COLS - 1) / COLS);
  const int n_active = __builtin_amdgcn_readfirstlane(rt.n_active);
  const int units = ncb_s + n_active * ncb;
  Tv* const act_sh = static_cast<Tv*>(a.act) + (int64_t)a.T * a.k * a.F;
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    if (unit < ncb_s) {
      dispatch(a.T, nullptr, nullptr, static_cast<const Tv*>(a.sh_gate),
               static_cast<const Tv*>(a.sh_up), (int64_t)unit * COLS, a.Fs, act_sh);
    } else {
      const int v = unit - ncb_s;
      const int e = __builtin_amdgcn_readfirstlane(rt.list[v / ncb]);
      const int base = __builtin_amdgcn_readfirstlane(rt.base[e]);
      const int m = __builtin_amdgcn_readfirstlane(__popcll(rt.mask[e]));
      const int64_t sl = __builtin_amdgcn_readfirstlane(a.slot ? a.slot[e] : e);
      dispatch(m, rt.row_token + base, rt.row_gate + base,
               static_cast<const Tv*>(a.w_gate) + sl * a.F * K,
               static_cast<const Tv*>(a.w_up) + sl * a.F * K, (int64_t)(v % ncb) * COLS, a.F,
               static_cast<Tv*>(a.act) + (int64_t)base * a.F);
    }
  }
}

// ---------------------------------------------------------------- down
// Block (x: 16 * NT columns, y: K part). The K blocks of all active experts and
// the shared ones form one sequence, which parts and waves cut into contiguous
// ranges; row t of the product is token t, zero where t is not the expert's.
template <typename Tv, int MT, int NT>
__global__ void __launch_bounds__(kLdThreads, 2)
ld_down_kernel(LdArgs a, int accumulate, float* __restrict__ partial, int32_t* __restrict__ count,
               Tv* __restrict__ y) {
  using LT = LdType<Tv>;
  constexpr int U = MT == 1 ? 8 / NT : MT == 2 ? 6 / NT : 4 / NT;
  __shared__ LdEntry ent[kLdExperts];
  __shared__ f32x4_t part[kLdWaves][MT][NT][kWave];
  __shared__ int s_last;
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane & 15, q4 = lane >> 4;
  const int n_ent = __builtin_amdgcn_readfirstlane(*a.n_entries);
  for (int q = threadIdx.x; q < n_ent; q += kLdThreads) ent[q] = a.entries[q];
  __syncthreads();
  const int64_t n0 = (int64_t)blockIdx.x * 16 * NT;
  const int nb = (int)((a.F + LT::KB - 1) / LT::KB), nbs = (int)((a.Fs + LT::KB - 1) / LT::KB);
  const int64_t total = (int64_t)n_ent * nb + nbs;
  const int64_t q_n = (int64_t)gridDim.y * kLdWaves, q_i = (int64_t)blockIdx.y * kLdWaves + wave;
  const int64_t lo = total * q_i / q_n, hi = total * (q_i + 1) / q_n;
  const uint32_t act_bytes = (uint32_t)(((int64_t)a.T * a.k * a.F + a.T * a.Fs) * sizeof(Tv));
  const rsrc_t rs_a = __builtin_amdgcn_make_buffer_rsrc(a.act, 0, (int)act_bytes, 0x00027000);
  const uint32_t w_chunk = (q4 + ((lane >> 3) & 1) * 4) * 16;
  f32x4_t acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // the place in the sequence: entry (n_ent: shared) and K block in it
  int en = nb > 0 ? (int)min(lo / nb, (int64_t)n_ent) : 0;
  int kb = (int)(lo - (int64_t)en * nb);
  rsrc_t rs[NT];
  uint32_t a_off[MT], row_bytes = 0;
  auto enter = [&]() {                           // descriptors of entry en
    const bool sh = en >= n_ent;
    const int64_t K = sh ? a.Fs : a.F;
    row_bytes = (uint32_t)(K * sizeof(Tv));
    uint64_t mask = ~0ull;
    int64_t sl = 0;
    uint32_t first = (uint32_t)((int64_t)a.T * a.k * a.F * sizeof(Tv));
    if (!sh) {
      const LdEntry& q = ent[en];
      mask = q.mask;
      sl = __builtin_amdgcn_readfirstlane(q.slot);
      first = (uint32_t)__builtin_amdgcn_readfirstlane(q.base) * row_bytes;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int t = 16 * i + r;
      const bool in = t < a.T && ((mask >> t) & 1);
      a_off[i] = in ? first + (uint32_t)__popcll(mask & ((1ull << t) - 1)) * row_bytes + q4 * 16
                    : kPastEnd;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      // a tile past H (the last block's second) re-reads the first, not stored
      const int64_t n = n0 + 16 * j < a.H ? n0 + 16 * j : n0;
      const int64_t rows = min(a.H - n, (int64_t)16);
      const Tv* const p = sh ? static_cast<const Tv*>(a.sh_down) + n * K
                             : static_cast<const Tv*>(a.w_down) + (sl * a.H + n) * K;
      rs[j] = __builtin_amdgcn_make_buffer_rsrc(const_cast<Tv*>(p), 0, (int)(rows * row_bytes),
                                                0x00027000);
    }
  };
  if (lo < hi) enter();
  for (int64_t g0 = lo; g0 < hi; g0 += U) {
    u32x4_t w[U][NT][2], x[U][MT][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (g0 + u >= hi) break;
      const uint32_t at = (uint32_t)kb * 128;
      const uint32_t w_off = (uint32_t)(lane & 7) * row_bytes + w_chunk;
      const bool w_in = at + w_chunk < row_bytes;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
          w[u][j][hh] = buf_load16<true>(rs[j], w_in ? w_off + hh * 8 * row_bytes : kPastEnd, at);
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const bool in = at + hh * 64 + q4 * 16 < row_bytes;
#pragma unroll
        for (int i = 0; i < MT; ++i)
          x[u][i][hh] = buf_load16<false>(rs_a, in && a_off[i] != kPastEnd ? a_off[i] + hh * 64 : kPastEnd, at);
      }
      if (++kb == (en >= n_ent ? nbs : nb) && g0 + u + 1 < hi) {
        ++en;
        kb = 0;
        enter();
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (g0 + u >= hi) break;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        u32x4_t w0, w1;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          w0[v] = ror8_into(w[u][j][0][v], w[u][j][1][v], true);
          w1[v] = ror8_into(w[u][j][1][v], w[u][j][0][v], false);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          LT::mfma(acc[i][j], x[u][i][0], w0);
          LT::mfma(acc[i][j], x[u][i][1], w1);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) part[wave][i][j][lane] = acc[i][j];
  __syncthreads();
  // a part's sums of one (row tile, column tile): 64 x 16 bytes
  const int64_t tiles = (int64_t)gridDim.x * MT * NT;
  auto slice = [&](int p, int i, int j) {
    return reinterpret_cast<f32x4_t*>(partial) +
           (p * tiles + (int64_t)blockIdx.x * MT * NT + i * NT + j) * kWave;
  };
  if (gridDim.y > 1) {
    for (int g = wave; g < MT * NT; g += kLdWaves) {
      const int i = g / NT, j = g % NT;
      f32x4_t s = part[0][i][j][lane];
#pragma unroll
      for (int w = 1; w < kLdWaves; ++w) s += part[w][i][j][lane];
      slice(blockIdx.y, i, j)[lane] = s;
    }
    // the last part to arrive adds them all, in part order
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicAdd(&count[blockIdx.x], 1) == (int)gridDim.y - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
  }
  for (int g = wave; g < MT * NT; g += kLdWaves) {
    const int i = g / NT, j = g % NT;
    f32x4_t s;
    if (gridDim.y > 1) {
      s = slice(0, i, j)[lane];
      for (int p = 1; p < (int)gridDim.y; ++p) s += slice(p, i, j)[lane];
    } else {
      s = part[0][i][j][lane];
#pragma unroll
      for (int w = 1; w < kLdWaves; ++w) s += part[w][i][j][lane];
    }
    const int64_t col = n0 + 16 * j + r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int t = 16 * i + 4 * q4 + q;
      if (t < a.T && col < a.H) {
        Tv* const o = y + t * a.H + col;
        *o = LT::put(accumulate ? s[q] + LT::get(*o) : s[q]);
      }
    }
  }
}

template <typename Tv, int MTMAX>
int ld_launch(const LdArgs& a, int accumulate, const LdLayout& lay, char* ws, void* y,
              hipStream_t st) {
  const int64_t cus = device_cu_count();
  const int64_t experts = std::min<int64_t>((int64_t)a.T * a.k, std::min(a.E, a.S));
  constexpr int NT = 1;
  const int64_t units = ceil_div(a.Fs, 16 * NT) + experts * ceil_div(a.F, 16 * NT);
  const unsigned grid = (unsigned)std::max<int64_t>(1, std::min(units, 2 * cus));
  ld_up_kernel<Tv, MTMAX, NT><<<dim3(grid), dim3(kLdThreads), 0, st>>>(a);
  MOE_CHECK_LAUNCH();
  ld_down_kernel<Tv, MTMAX, kDownTiles>
      <<<dim3((unsigned)lay.col_tiles, (unsigned)lay.parts), dim3(kLdThreads), 0, st>>>(
          a, accumulate, reinterpret_cast<float*>(ws + lay.part),
          reinterpret_cast<int32_t*>(ws + lay.count), static_cast<Tv*>(y));
  MOE_CHECK_LAUNCH();
  return MOE_OK;
}

template <typename Tv>
int ld_run(LdArgs a, const void* w_router, const float* bias, int32_t bias_mode, int accumulate,
           const LdLayout& lay, char* ws, void* y, hipStream_t st) {
  ld_logits_kernel<Tv><<<dim3((unsigned)a.E, (unsigned)ceil_div(a.T, kLdWaves)), dim3(kLdThreads),
                         0, st>>>(static_cast<const Tv*>(a.x), static_cast<const Tv*>(w_router),
                                  a.T, a.H, a.E, bias, bias_mode,
                                  reinterpret_cast<double*>(ws + lay.z),
                                  reinterpret_cast<int32_t*>(ws + lay.count), lay.col_tiles);
  MOE_CHECK_LAUNCH();
  if (a.T <= 16) return ld_launch<Tv, 1>(a, accumulate, lay, ws, y, st);
  if (a.T <= 32) return ld_launch<Tv, 2>(a, accumulate, lay, ws, y, st);
  return ld_launch<Tv, 4>(a, accumulate, lay, ws, y, st);
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
  a.z = reinterpret_cast<const double*>(ws + lay.z);
  a.act = ws + lay.act;
  a.entries = reinterpret_cast<LdEntry*>(ws + lay.entries);
  a.n_entries = reinterpret_cast<int32_t*>(ws + lay.meta);
  a.topk_idx = topk_idx;
  a.topk_w = topk_w;
  a.incomplete = incomplete;
  hipStream_t st = as_stream(stream);
  return dtype == MOE_BF16
             ? ld_run<uint16_t>(a, w_router, bias, bias_mode, accumulate, lay, ws, y, st)
             : ld_run<float>(a, w_router, bias, bias_mode, accumulate, lay, ws, y, st);
}
