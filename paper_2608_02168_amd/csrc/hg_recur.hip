// Gated linear recurrence over channels: whole histories forward and backward,
// and single tokens.
//
//   a_t = exp(l sigmoid(r_t)),  l = -rate softplus(decay)
//   h_t = a_t h_{t-1} + u_t,    u_t = sqrt(1 - a_t^2) sigmoid(i_t) x_t
// backward, with c_t = a_t g_t what the gradient g_t of h_t passes to token t-1:
//   c_t = a_t c_{t+1} + a_t dh_t,   g_t = dh_t + c_{t+1}
// Both are first-order recurrences y' = A y + B, whose steps compose:
// (A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2).
//
// A thread has four channels and K tokens in a row.  It composes its tokens' steps
// in registers, the four runs of a wave (16 threads side by side) compose by
// shuffles, the waves of a block through LDS; then each thread walks its tokens
// again from the value that reaches it.  So a block takes 16 K tokens of 64 channels
// at a time, and every value is read and written once.  Many sequences: a wave
// (WAVE: no barrier) or a block walks each.  Few: a block for each tile, all at once,
// and the tiles' steps compose through memory (k_recur_chain_*).
//
// The gates are a published recurrence's (S. De and others, 2024, arXiv 2402.19427); that
// tiles publish their composed steps and form their prefix from those before is the
// one-pass scan of D. Merrill and M. Garland, 2016.
//
// Bound by HBM and by the vector instructions at once: 49 issue slots a value forward, six
// instructions of them transcendental, are 83 us for 67M values on this chip, their 8
// bytes 103 us at the 5.2 TB/s of a large copy (one pass over both: 128 us).
//
// The last four channels of a row whose width is no multiple of four are taken
// by a thread that starts earlier: two threads then compute and write the same
// values of the same addresses.
#include <cmath>
#include <type_traits>

#include "hg_rows4.h"

namespace hg {
namespace {

constexpr int V = 4;             // channels of a thread
constexpr int CL = 16;           // threads side by side
constexpr int TW = 64 / CL;      // runs of tokens in a wave
constexpr int kSlab = CL * V;    // channels of a block
constexpr int kNW = 4;           // waves of a block
constexpr float kLog2e = 1.4426950408889634f;

struct RecurArgs {
  Rows x, r, i, h, dh;   // inputs (h: the forward's output)
  Rows dx, dr, di;
  const float* decay;
  const int32_t* lens;
  const float* s_in;     // state, in the backward dstate_out
  const float* s_first;  // backward: the forward's state
  float* s_out;
  float* part;           // [blocks of a slab][width] sums of dlog sigmoid(r), or null
  int64_t t;
  int32_t batch, width, slabs;
  float rate;
};

template <class T>
using Quad = Vec<T, V>;

// sigmoid(z) from e = 2^(-z log2 e), and sigmoid(-z) by its own size: 1 - sigmoid(z) has
// no digits left from z = 17 on.  (Where e is infinite the sigmoid is 0, and so is
// what the backward multiplies the other with: any finite value will do.)
__device__ __forceinline__ float exp_of(float z) { return __builtin_amdgcn_exp2f(-kLog2e * z); }
__device__ __forceinline__ float sigm_of(float e) { return __builtin_amdgcn_rcpf(1.f + e); }
__device__ __forceinline__ float rest_of_sigm(float e, float s) { return fminf(e, 3.4e38f) * s; }
__device__ __forceinline__ float sigm(float z) { return sigm_of(exp_of(z)); }

// rate softplus(decay) log2 e: the factor is 2^(-that sigmoid(r)).  Finite, so that it is
// 0 times sigmoid(r) = 0.
__device__ __forceinline__ float slope_of(float decay, float rate) {
  const float v = rate * kLog2e * (fmaxf(decay, 0.f) + log1pf(expf(-fabsf(decay))));
  return v == INFINITY ? 3.4e38f : v;
}

// 1 - a^2 for a = 2^l: near a = 1 by the series of 1 - e^y, y = 2 l ln 2, to y^6
// (relative error 5e-8 at y = -1/4, where 1 - a a has 4e-7).  bfloat16 rows take it
// too: the states are float32.
__device__ __forceinline__ float rest_of(float l, float a) {
  constexpr float y = 1.3862943611198906f;  // y / l
  float p = fmaf(l, -y * y * y * y * y * y / 720.f, -y * y * y * y * y / 120.f);
  p = fmaf(l, p, -y * y * y * y / 24.f);
  p = fmaf(l, p, -y * y * y / 6.f);
  p = fmaf(l, p, -y * y / 2.f);
  p = fmaf(l, p, -y);
  return l > -0.25f / y ? l * p : fmaf(-a, a, 1.f);
}

// The steps of the runs before this thread's in its wave (sign 1: the ranks below), and
// of the whole wave.
struct Step {
  float a[V], b[V];
};
__device__ __forceinline__ void compose_wave(Step& s, Step& before, int rank) {
#pragma unroll
  for (int o = 1; o < TW; o *= 2) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float pa = __shfl_up(s.a[j], o * CL, 64), pb = __shfl_up(s.b[j], o * CL, 64);
      if (rank >= o) {
        s.b[j] = fmaf(s.a[j], pb, s.b[j]);
        s.a[j] *= pa;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float pa = __shfl_up(s.a[j], CL, 64), pb = __shfl_up(s.b[j], CL, 64);
    before.a[j] = rank ? pa : 1.f;
    before.b[j] = rank ? pb : 0.f;
  }
}

// y: the value that reaches the tile; becomes the one that leaves it.  Returns in
// `at` the value that reaches this thread's run.  lds: this tile's [NW][2][64].
template <bool WAVE>
__device__ __forceinline__ void compose(Step& s, float (&y)[V], float (&at)[V], float* lds, int wave, int rank, int col) {
  Step before;
  compose_wave(s, before, rank);
  if constexpr (WAVE) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      at[j] = fmaf(before.a[j], y[j], before.b[j]);
      const int last = (TW - 1) * CL + col;
      y[j] = fmaf(__shfl(s.a[j], last, 64), y[j], __shfl(s.b[j], last, 64));
    }
  } else {
    if (rank == TW - 1) {
      *reinterpret_cast<f32x4*>(lds + wave * 2 * kSlab + col * V) = f32x4{s.a[0], s.a[1], s.a[2], s.a[3]};
      *reinterpret_cast<f32x4*>(lds + wave * 2 * kSlab + kSlab + col * V) = f32x4{s.b[0], s.b[1], s.b[2], s.b[3]};
    }
    __syncthreads();
    float w[V];
#pragma unroll
    for (int q = 0; q < kNW; ++q) {
#pragma unroll
      for (int j = 0; j < V; ++j) w[j] = q == wave ? y[j] : w[j];
      const f32x4 qa = *reinterpret_cast<const f32x4*>(lds + q * 2 * kSlab + col * V);
      const f32x4 qb = *reinterpret_cast<const f32x4*>(lds + q * 2 * kSlab + kSlab + col * V);
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = fmaf(qa[j], y[j], qb[j]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) at[j] = fmaf(before.a[j], w[j], before.b[j]);
  }
}

// What a block (WAVE: a wave) works on.  All but the channels is the same in a wave.
struct Place {
  int64_t b, t_end, out_end;  // its sequence, whose rows past t_end are zeros up to out_end
  int32_t c0;                 // first channel of the thread
  bool on;                    // no thread before has the same channels
};
__device__ __forceinline__ int64_t len_of(const RecurArgs& a, int64_t b) {
  if (!a.lens) return a.t;
  const int32_t n = a.lens[b];
  return n < 0 ? 0 : (n < a.t ? n : a.t);
}
// A thread's channels: the last ones of a row start at width - V.
__device__ __forceinline__ void channels_of(const RecurArgs& a, int slab, int col, Place& p) {
  const int c = slab * kSlab + col * V;
  p.on = c < a.width;
  p.c0 = c < a.width - V ? c : a.width - V;
}
template <bool WAVE>
__device__ __forceinline__ Place place_of(const RecurArgs& a, int wave, int col) {
  Place p;
  const uint32_t id = blockIdx.x, rest = id / (uint32_t)a.slabs;
  p.b = WAVE ? (int64_t)rest * kNW + wave : rest;
  channels_of(a, (int)(id - rest * (uint32_t)a.slabs), col, p);
  p.t_end = p.b < a.batch ? len_of(a, p.b) : 0;
  p.out_end = a.t;
  return p;
}

// One operand's rows of a sequence: an address that is the same in a wave and a
// thread's 32-bit offset from it, so that a row costs no vector instruction but its
// load (Off 32 bits: a block's tile is below 2^32 bytes, kMaxToken).
template <class T, class Off = uint32_t>
struct Stream {
  const char* base;  // token 0
  int64_t row;       // bytes between tokens
  Off off;           // of the thread, from the tile's first token
  __device__ __forceinline__ Stream(const Rows& x, const Place& p, Off skip)
      : base(static_cast<const char*>(x.p) + p.b * x.sb * (int64_t)sizeof(T)), row(x.st * (int64_t)sizeof(T)),
        off(skip * (Off)(x.st * (int64_t)sizeof(T)) + (Off)p.c0 * (Off)sizeof(T)) {}
  // the thread's token k of the tile from token ts on
  __device__ __forceinline__ T* at(int64_t ts, int k) const {
    return reinterpret_cast<T*>(const_cast<char*>(base + (ts + k) * row + off));
  }
};

// K rows of one operand, the thread's tokens t .. of the tile from ts on; FULL: all
// are inside, else those in [lo, hi) are read.
template <class T, int K, bool FULL, class Off>
__device__ __forceinline__ void load(typename Quad<T>::raw (&w)[K], const Stream<T, Off>& x, int64_t ts, int64_t t, int64_t lo,
                                     int64_t hi) {
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (FULL || (t + k >= lo && t + k < hi)) w[k] = Quad<T>::load(x.at(ts, k));
}

// The rows past a sequence's end as zeros.
template <class T>
__device__ __forceinline__ void zero_rows(const Rows& x, const Place& p, int rank, int ranks) {
  const float z[V] = {0.f, 0.f, 0.f, 0.f};
  T* o = static_cast<T*>(x.p) + p.b * x.sb + p.c0;
  if (p.on)
    for (int64_t t = p.t_end + rank; t < p.out_end; t += ranks) Quad<T>::put(o + t * x.st, z);
}

template <bool B>
using Bool = std::integral_constant<bool, B>;

__device__ __forceinline__ void load_state(const float* s, const RecurArgs& a, const Place& p, float (&y)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) y[j] = s ? s[p.b * a.width + p.c0 + j] : 0.f;
}

template <class T, int K, bool WAVE>
__global__ void __launch_bounds__(kNW * 64) k_recur_fwd(const RecurArgs a) {
  __shared__ __align__(16) float lds[WAVE ? 4 : 2 * kNW * 2 * kSlab];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane % CL, rank = lane / CL;
  constexpr int kTile = (WAVE ? 1 : kNW) * TW * K;
  const Place p = place_of<WAVE>(a, wave, col);
  if (WAVE && p.b >= a.batch) return;
  const int run = WAVE ? rank : wave * TW + rank;
  float slope[V], y[V];
#pragma unroll
  for (int j = 0; j < V; ++j) slope[j] = -slope_of(a.decay[p.c0 + j], a.rate);
  load_state(a.s_in, a, p, y);
  const Stream<T> sx(a.x, p, run * K), sr(a.r, p, run * K), si(a.i, p, run * K), sh(a.h, p, run * K);
  typename Quad<T>::raw rx[K] = {}, rr[K] = {}, ri[K] = {};
  auto fetch = [&](auto full, int64_t ts) {
    constexpr bool FULL = decltype(full)::value;
    load<T, K, FULL>(rr, sr, ts, ts + run * K, 0, p.t_end);
    load<T, K, FULL>(ri, si, ts, ts + run * K, 0, p.t_end);
    load<T, K, FULL>(rx, sx, ts, ts + run * K, 0, p.t_end);
  };
  int odd = 0;
  auto tile = [&](auto full, int64_t ts) {
    constexpr bool FULL = decltype(full)::value;
    const int64_t t0 = ts + run * K;
    float fa[K][V], fu[K][V];
    Step s;
#pragma unroll
    for (int j = 0; j < V; ++j) s.a[j] = 1.f, s.b[j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool in = FULL || t0 + k < p.t_end;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float l = slope[j] * sigm(Quad<T>::get(rr[k], j));
        const float f = __builtin_amdgcn_exp2f(l);
        const float u = __builtin_amdgcn_sqrtf(rest_of(l, f)) * sigm(Quad<T>::get(ri[k], j)) * Quad<T>::get(rx[k], j);
        fa[k][j] = in ? f : 1.f;
        fu[k][j] = in ? u : 0.f;
        s.a[j] *= fa[k][j];
        s.b[j] = fmaf(fa[k][j], s.b[j], fu[k][j]);
      }
    }
    if (ts + 2 * kTile <= p.t_end) {
      fetch(Bool<true>{}, ts + kTile);
    } else if (ts + kTile < p.t_end) {
      fetch(Bool<false>{}, ts + kTile);
    }
    float at[V];
    compose<WAVE>(s, y, at, lds + (WAVE ? 0 : odd * kNW * 2 * kSlab), wave, rank, col);
    odd ^= 1;
    if (p.on) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int j = 0; j < V; ++j) at[j] = fmaf(fa[k][j], at[j], fu[k][j]);
        if (FULL || t0 + k < p.t_end) Quad<T>::put(sh.at(ts, k), at);
      }
    }
  };
  int64_t ts = 0;
  if (ts + kTile <= p.t_end) {
    fetch(Bool<true>{}, ts);
  } else {
    fetch(Bool<false>{}, ts);
  }
  for (; ts + kTile <= p.t_end; ts += kTile) tile(Bool<true>{}, ts);
  if (ts < p.t_end) tile(Bool<false>{}, ts);
  zero_rows<T>(a.h, p, run, WAVE ? TW : kNW * TW);
  if (a.s_out && p.on && run == 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) a.s_out[p.b * a.width + p.c0 + j] = y[j];
  }
}

// The gradients at one token, and what it adds to the sums; at: the gradient that
// reaches h from the token after, becomes the one that this token passes on.  fe: the
// exponential of the gate r, from which its sigmoid is formed again (as many registers
// as the sigmoid, and the derivative keeps its digits).  The empty asm keeps the compiler
// from holding the sigmoids and the unpacked dh as well (bfloat16 tiles 240 registers, 283
// and one wave a SIMD without).
template <class T>
__device__ __forceinline__ void grads_of(const float (&slope)[V], const float (&fe)[V], const float (&fa)[V],
                                         typename Quad<T>::raw rg, const typename Quad<T>::raw& ri,
                                         const typename Quad<T>::raw& rx, const float (&hb)[V], float (&at)[V], float (&sum)[V],
                                         float (&vx)[V], float (&vi)[V], float (&vr)[V]) {
  asm("" : "+v"(rg));
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float er = fe[j];
    asm("" : "+v"(er));
    const float s = sigm_of(er), f = fa[j], l = slope[j] * s, g = Quad<T>::get(rg, j) + at[j];
    at[j] = f * g;
    // (1 - a^2 below the smallest normal number, whose root the hardware does not take, is zero)
    const float m = rest_of(l, f), iq = m >= 0x1p-126f ? __builtin_amdgcn_rsqf(m) : 0.f, q = m * iq;
    const float ei = exp_of(Quad<T>::get(ri, j)), sg = sigm_of(ei), x = Quad<T>::get(rx, j), gs = g * sg;
    vx[j] = gs * q;
    vi[j] = vx[j] * x * rest_of_sigm(ei, sg);
    const float dl = f * fmaf(g, hb[j], -gs * iq * f * x);  // (iq first: where it is zero, no product of g and x)
    sum[j] = fmaf(dl, s, sum[j]);
    vr[j] = dl * (l * 0.69314718055994531f) * rest_of_sigm(er, s);
  }
}

// A block's sums of its runs, in order, as row `at` of the partial sums.
__device__ __forceinline__ void block_sums(const RecurArgs& a, const float (&sum)[V], float* all, int run, int col, int slab,
                                           int64_t at) {
#pragma unroll
  for (int j = 0; j < V; ++j) all[run * kSlab + col * V + j] = sum[j];
  __syncthreads();
  for (int c = threadIdx.x; c < kSlab; c += kNW * 64) {
    const int ch = slab * kSlab + c;
    if (ch >= a.width) continue;
    // the thread that has channel ch: the last ones start at width - V
    const int own = c / V, c0 = slab * kSlab + own * V, shift = c0 < a.width - V ? 0 : c0 - (a.width - V);
    float s = 0.f;
    for (int q = 0; q < kNW * TW; ++q) s += all[q * kSlab + c + shift];
    a.part[at * a.width + ch] = s;
  }
}

// WAVE: a wave takes every `stride`-th sequence from its own on, so that the
// partial sums of ddecay are few.
template <class T, int K, bool WAVE>
__global__ void __launch_bounds__(kNW * 64) k_recur_bwd(const RecurArgs a, int32_t stride) {
  __shared__ __align__(16) float lds[2 * kNW * 2 * kSlab];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane % CL, rank = lane / CL;
  constexpr int kRuns = (WAVE ? 1 : kNW) * TW, kTile = kRuns * K;
  const int run = WAVE ? rank : wave * TW + rank, skip = (kRuns - 1 - run) * K;  // the first run is the tile's last
  Place p = place_of<WAVE>(a, wave, col);
  float slope[V], sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    slope[j] = -slope_of(a.decay[p.c0 + j], a.rate);
    sum[j] = 0.f;
  }
  for (; p.b < a.batch; p.b += stride) {
    if (WAVE) p.t_end = len_of(a, p.b);
    float y[V];
    load_state(a.s_in, a, p, y);
    const Stream<T> sx(a.x, p, skip), sr(a.r, p, skip), si(a.i, p, skip), sh(a.h, p, skip), sg(a.dh, p, skip), ox(a.dx, p, skip),
        orr(a.dr, p, skip), oi(a.di, p, skip);
    typename Quad<T>::raw rx[K] = {}, rr[K] = {}, ri[K] = {}, rh[K] = {}, rg[K] = {};
    // the tile of tokens ts .. ts + kTile - 1 (row k of rh: h before the thread's token k); FULL: it begins after token 0
    auto fetch = [&](auto full, int64_t ts) {
      constexpr bool FULL = decltype(full)::value;
      load<T, K, FULL>(rr, sr, ts, ts + skip, 0, p.t_end);
      load<T, K, FULL>(rg, sg, ts, ts + skip, 0, p.t_end);
      load<T, K, FULL>(ri, si, ts, ts + skip, 0, p.t_end);
      load<T, K, FULL>(rx, sx, ts, ts + skip, 0, p.t_end);
      load<T, K, FULL>(rh, sh, ts - 1, ts - 1 + skip, 0, p.t_end);
    };
    int odd = 0;
    auto tile = [&](auto full, int64_t ts) {
      constexpr bool FULL = decltype(full)::value;
      const int64_t t0 = ts + skip;
      float fe[K][V], fa[K][V];
      Step s;
#pragma unroll
      for (int j = 0; j < V; ++j) s.a[j] = 1.f, s.b[j] = 0.f;
#pragma unroll
      for (int k = K - 1; k >= 0; --k) {
        const bool in = FULL || t0 + k >= 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          fe[k][j] = exp_of(Quad<T>::get(rr[k], j));
          const float f = __builtin_amdgcn_exp2f(slope[j] * sigm_of(fe[k][j]));
          fa[k][j] = in ? f : 1.f;
          s.b[j] = fa[k][j] * (s.b[j] + (in ? Quad<T>::get(rg[k], j) : 0.f));
          s.a[j] *= fa[k][j];
        }
      }
      float at[V];
      compose<WAVE>(s, y, at, lds + (WAVE ? 0 : odd * kNW * 2 * kSlab), wave, rank, col);
      odd ^= 1;
#pragma unroll
      for (int k = K - 1; k >= 0; --k) {
        if (!FULL && t0 + k < 0) continue;
        float hb[V], vx[V], vi[V], vr[V];
#pragma unroll
        for (int j = 0; j < V; ++j) hb[j] = Quad<T>::get(rh[k], j);
        if (!FULL && t0 + k == 0) load_state(a.s_first, a, p, hb);
        grads_of<T>(slope, fe[k], fa[k], rg[k], ri[k], rx[k], hb, at, sum, vx, vi, vr);
        if (p.on) {
          Quad<T>::put(ox.at(ts, k), vx);
          Quad<T>::put(oi.at(ts, k), vi);
          Quad<T>::put(orr.at(ts, k), vr);
        }
      }
      // the tile before; one that holds token 0 is not full (its h before comes from the state)
      if (ts - kTile > 0) {
        fetch(Bool<true>{}, ts - kTile);
      } else if (ts > 0) {
        fetch(Bool<false>{}, ts - kTile);
      }
    };
    int64_t ts = p.t_end - kTile;
    if (ts > 0) {
      fetch(Bool<true>{}, ts);
    } else {
      fetch(Bool<false>{}, ts);
    }
    for (; ts > 0; ts -= kTile) tile(Bool<true>{}, ts);
    if (ts + kTile > 0) tile(Bool<false>{}, ts);
    const int ranks = WAVE ? TW : kNW * TW;
    zero_rows<T>(a.dx, p, run, ranks);
    zero_rows<T>(a.di, p, run, ranks);
    zero_rows<T>(a.dr, p, run, ranks);
    if (a.s_out && p.on && run == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) a.s_out[p.b * a.width + p.c0 + j] = y[j];
    }
    if (!WAVE) break;
  }
  if (!a.part) return;
  __syncthreads();
  static_assert(kNW * TW * kSlab <= 2 * kNW * 2 * kSlab, "the sums fit the block's LDS");
  const uint32_t rest = blockIdx.x / (uint32_t)a.slabs;
  block_sums(a, sum, lds, wave * TW + rank, col, (int)(blockIdx.x - rest * (uint32_t)a.slabs), rest);
}

// ---- one pass over few long histories ------------------------------------------------
// A block has one tile of 64 channels.  Blocks take tickets, tile by tile of all
// sequences, publish their tile's composed step (A, B) and form the value y that
// reaches it from the steps of the tiles before in its group of kGroup and the value
// that reaches the group, which the last block of the group before publishes.  The
// order of every product is fixed, so results do not depend on timing.
//
// A published word is its own flag: the words are all ones (a NaN that no step is
// stored as) before the launch, and are stored and read whole, at device scope.  A
// block waits for blocks of lower tickets only, which have started, and which publish
// their step before they wait for anything: every wait ends.  (Two calls at once on one
// workspace clear each other's words.  A wait that has looked kTries times, seconds,
// writes NaN for its word, so that such calls end too, with NaN; a ticket past the last
// tile ends its block.)
constexpr int kGroup = 32;  // (16 and 64: within 1 %)
constexpr uint32_t kNone = 0xFFFFFFFFu;

struct Chain {
  uint64_t* step;    // [pairs][tiles][64]: A, B
  uint32_t* value;   // [pairs][groups][64]: y that reaches a group (of group 0: not used)
  uint32_t* ticket;
  int32_t tiles, groups;
  uint32_t pairs;
};

__device__ __forceinline__ uint32_t word_of(float v) {
  const uint32_t u = __float_as_uint(v);
  return u == kNone ? 0x7FC00000u : u;
}
__device__ __forceinline__ uint64_t peek(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t peek(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

constexpr int kTries = 1 << 22;
__device__ __forceinline__ uint32_t flag_of(uint64_t w) { return (uint32_t)w; }
__device__ __forceinline__ uint32_t flag_of(uint32_t w) { return w; }
// The word at p once it is there; w: as it was read before.
template <class W>
__device__ __forceinline__ W await(W* p, W w) {
  for (int n = 0; flag_of(w) == kNone; ++n) {
    if (n == kTries) {
      w = sizeof(W) == 8 ? (W)0x7FC000007FC00000ull : (W)0x7FC00000u;
      __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      break;
    }
    __builtin_amdgcn_s_sleep(1);
    w = peek(p);
  }
  return w;
}

struct ChainLds {
  float wave[kNW][2][kSlab];  // the waves' steps
  float far[kNW][2][kSlab];   // steps of the tiles before, by wave
  float y[kSlab];             // the value that reaches the tile
  uint32_t ticket;
};

// The block's tile: its ticket's place, n counted in the walk's order.
__device__ __forceinline__ uint32_t take_ticket(const Chain& q, ChainLds& sh) {
  if (threadIdx.x == 0) sh.ticket = atomicAdd(q.ticket, 1u);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(sh.ticket);
}

// From the threads' steps s: `at`, the value that reaches this thread's run.  Lane l of
// a wave has channel l of the slab in between; y0: the value that reaches the first
// tile, of that channel; last: no tile after this one needs its value, which `out` has.
__device__ __forceinline__ void chain(Step& s, float (&at)[V], float& out, const Chain& q, ChainLds& sh, uint32_t pair, int n,
                                      bool last, float y0, int wave, int rank, int col) {
  const int lane = threadIdx.x & 63;
  Step before;
  compose_wave(s, before, rank);
  if (rank == TW - 1) {
    *reinterpret_cast<f32x4*>(&sh.wave[wave][0][col * V]) = f32x4{s.a[0], s.a[1], s.a[2], s.a[3]};
    *reinterpret_cast<f32x4*>(&sh.wave[wave][1][col * V]) = f32x4{s.b[0], s.b[1], s.b[2], s.b[3]};
  }
  __syncthreads();
  float ta = 1.f, tb = 0.f;  // the tile's step
#pragma unroll
  for (int w = 0; w < kNW; ++w) {
    const float a = sh.wave[w][0][lane], b = sh.wave[w][1][lane];
    tb = fmaf(a, tb, b);
    ta *= a;
  }
  const int group = n / kGroup, r = n - group * kGroup;
  uint64_t* steps = q.step + ((int64_t)pair * q.tiles + (n - r)) * kSlab + lane;
  if (wave == 0 && r != kGroup - 1 && !last)
    __hip_atomic_store(steps + (int64_t)r * kSlab, (uint64_t)__float_as_uint(tb) << 32 | word_of(ta), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  // this wave's share of the tiles before in the group, then the value that reaches the group
  constexpr int PER = kGroup / kNW;
  float fa = 1.f, fb = 0.f;
  {
    uint64_t w[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (wave * PER + k < r) w[k] = peek(steps + (int64_t)(wave * PER + k) * kSlab);
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (wave * PER + k < r) {
        w[k] = await(steps + (int64_t)(wave * PER + k) * kSlab, w[k]);
        const float a = __uint_as_float((uint32_t)w[k]), b = __uint_as_float((uint32_t)(w[k] >> 32));
        fb = fmaf(a, fb, b);
        fa *= a;
      }
  }
  sh.far[wave][0][lane] = fa;
  sh.far[wave][1][lane] = fb;
  __syncthreads();
  if (wave == 0) {
    float y = y0;
    if (group > 0) {
      uint32_t* v = q.value + ((int64_t)pair * q.groups + group) * kSlab + lane;
      y = __uint_as_float(await(v, peek(v)));
    }
#pragma unroll
    for (int w = 0; w < kNW; ++w) y = fmaf(sh.far[w][0][lane], y, sh.far[w][1][lane]);
    out = fmaf(ta, y, tb);
    if (r == kGroup - 1 && !last)
      __hip_atomic_store(q.value + ((int64_t)pair * q.groups + group + 1) * kSlab + lane, word_of(out), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    sh.y[lane] = y;
  }
  __syncthreads();
  f32x4 y = *reinterpret_cast<const f32x4*>(&sh.y[col * V]);
  for (int w = 0; w < wave; ++w) {
    const f32x4 qa = *reinterpret_cast<const f32x4*>(&sh.wave[w][0][col * V]);
    const f32x4 qb = *reinterpret_cast<const f32x4*>(&sh.wave[w][1][col * V]);
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = fmaf(qa[j], y[j], qb[j]);
  }
#pragma unroll
  for (int j = 0; j < V; ++j) at[j] = fmaf(before.a[j], y[j], before.b[j]);
}

// The channel that lane l has in chain().
__device__ __forceinline__ int channel_of(const RecurArgs& a, int slab, int lane) {
  const int c = slab * kSlab + (lane & ~(V - 1));
  return (c < a.width - V ? c : a.width - V) + (lane & (V - 1));
}

// A block's rows past the sequence's end, of its own stretch of the t tokens.
template <class T, int TILE>
__device__ __forceinline__ void zero_stretch(const RecurArgs& a, const Rows& x, Place p, int64_t len, int n, int run) {
  p.t_end = (int64_t)n * TILE > len ? (int64_t)n * TILE : len;
  p.out_end = (int64_t)(n + 1) * TILE < a.t ? (int64_t)(n + 1) * TILE : a.t;
  zero_rows<T>(x, p, run, kNW * TW);
}

// Gates r of rows that no token has: sigmoid(-inf) = 0, so that their factor is 1 and,
// with x = 0 or dh = 0, their step leaves the value as it is, with no select a value
// (65521 bfloat16 tokens of 1024 channels 137 us, 143 with selects, both 12 tokens a thread).
template <class T, int K>
__device__ __forceinline__ void no_token(typename Quad<T>::raw (&r)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k)
    if constexpr (sizeof(T) == 4) {
      r[k] = -INFINITY;
    } else {
      r[k] = 0xFF80FF80u;
    }
}
template <class T, int K>
__global__ void __launch_bounds__(kNW * 64) k_recur_chain_fwd(const RecurArgs a, const Chain q) {
  __shared__ ChainLds sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane % CL, rank = lane / CL;
  constexpr int kTile = kNW * TW * K;
  const uint32_t ticket = take_ticket(q, sh), n = ticket / q.pairs, pair = ticket - n * q.pairs;
  if (n >= (uint32_t)q.tiles) return;
  const int slab = (int)(pair % (uint32_t)a.slabs), run = wave * TW + rank;
  Place p;
  p.b = pair / (uint32_t)a.slabs;
  channels_of(a, slab, col, p);
  const int64_t len = len_of(a, p.b), ts = (int64_t)n * kTile, t0 = ts + run * K;
  const int64_t state_at = p.b * a.width + channel_of(a, slab, lane);
  if (ts < len) {
    const Stream<T> sx(a.x, p, run * K), sr(a.r, p, run * K), si(a.i, p, run * K), so(a.h, p, run * K);
    typename Quad<T>::raw rx[K] = {}, rr[K], ri[K] = {};
    no_token<T>(rr);
    const bool whole = ts + kTile <= len;
    if (whole) {
      load<T, K, true>(rr, sr, ts, t0, 0, len);
      load<T, K, true>(ri, si, ts, t0, 0, len);
      load<T, K, true>(rx, sx, ts, t0, 0, len);
    } else {
      load<T, K, false>(rr, sr, ts, t0, 0, len);
      load<T, K, false>(ri, si, ts, t0, 0, len);
      load<T, K, false>(rx, sx, ts, t0, 0, len);
    }
    float slope[V], fa[K][V], fu[K][V], at[V], y0 = 0.f, out = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) slope[j] = -slope_of(a.decay[p.c0 + j], a.rate);
    if (n < kGroup && a.s_in) y0 = a.s_in[state_at];  // (it reaches group 0)
    Step s;
#pragma unroll
    for (int j = 0; j < V; ++j) s.a[j] = 1.f, s.b[j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float l = slope[j] * sigm(Quad<T>::get(rr[k], j));
        const float f = __builtin_amdgcn_exp2f(l);
        const float u = __builtin_amdgcn_sqrtf(rest_of(l, f)) * sigm(Quad<T>::get(ri[k], j)) * Quad<T>::get(rx[k], j);
        fa[k][j] = f;
        fu[k][j] = u;
        s.a[j] *= fa[k][j];
        s.b[j] = fmaf(fa[k][j], s.b[j], fu[k][j]);
      }
    }
    const bool last = ts + kTile >= len;
    chain(s, at, out, q, sh, pair, (int)n, last, y0, wave, rank, col);
    if (p.on) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int j = 0; j < V; ++j) at[j] = fmaf(fa[k][j], at[j], fu[k][j]);
        if (whole || t0 + k < len) Quad<T>::put(so.at(ts, k), at);
      }
    }
    if (last && a.s_out && wave == 0) a.s_out[state_at] = out;
  } else if (n == 0 && a.s_out && wave == 0) {
    a.s_out[state_at] = a.s_in ? a.s_in[state_at] : 0.f;  // no tokens
  }
  zero_stretch<T, kTile>(a, a.h, p, len, (int)n, run);
}

template <class T, int K>
__global__ void __launch_bounds__(kNW * 64) k_recur_chain_bwd(const RecurArgs a, const Chain q) {
  __shared__ ChainLds sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane % CL, rank = lane / CL;
  constexpr int kRuns = kNW * TW, kTile = kRuns * K;
  const uint32_t ticket = take_ticket(q, sh), n = ticket / q.pairs, pair = ticket - n * q.pairs;
  if (n >= (uint32_t)q.tiles) return;
  const int slab = (int)(pair % (uint32_t)a.slabs), run = wave * TW + rank, skip = (kRuns - 1 - run) * K;
  Place p;
  p.b = pair / (uint32_t)a.slabs;
  channels_of(a, slab, col, p);
  const int64_t len = len_of(a, p.b), ts = len - (int64_t)(n + 1) * kTile, t0 = ts + skip;  // the tiles end at the last token
  const int64_t state_at = p.b * a.width + channel_of(a, slab, lane);
  float sum[V] = {0.f, 0.f, 0.f, 0.f};
  if (ts + kTile > 0) {
    const Stream<T> sx(a.x, p, skip), sr(a.r, p, skip), si(a.i, p, skip), sh1(a.h, p, skip), sg(a.dh, p, skip), ox(a.dx, p, skip),
        orr(a.dr, p, skip), oi(a.di, p, skip);
    typename Quad<T>::raw rx[K] = {}, rr[K], ri[K] = {}, rh[K] = {}, rg[K] = {};
    no_token<T>(rr);
    const bool whole = ts > 0;  // (token 0's h before comes from the state)
    const auto fetch = [&](auto full) {
      constexpr bool FULL = decltype(full)::value;
      load<T, K, FULL>(rr, sr, ts, t0, 0, len);
      load<T, K, FULL>(rg, sg, ts, t0, 0, len);
      load<T, K, FULL>(ri, si, ts, t0, 0, len);
      load<T, K, FULL>(rx, sx, ts, t0, 0, len);
      load<T, K, FULL>(rh, sh1, ts - 1, t0 - 1, 0, len);
    };
    if (whole) {
      fetch(Bool<true>{});
    } else {
      fetch(Bool<false>{});
    }
    float slope[V], fe[K][V], fa[K][V], at[V], y0 = 0.f, out = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) slope[j] = -slope_of(a.decay[p.c0 + j], a.rate);
    if (n < kGroup && a.s_in) y0 = a.s_in[state_at];  // (it reaches group 0)
    Step s;
#pragma unroll
    for (int j = 0; j < V; ++j) s.a[j] = 1.f, s.b[j] = 0.f;
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        fe[k][j] = exp_of(Quad<T>::get(rr[k], j));
        const float f = __builtin_amdgcn_exp2f(slope[j] * sigm_of(fe[k][j]));
        fa[k][j] = f;
        s.b[j] = fa[k][j] * (s.b[j] + Quad<T>::get(rg[k], j));
        s.a[j] *= fa[k][j];
      }
    }
    const bool last = ts <= 0;
    chain(s, at, out, q, sh, pair, (int)n, last, y0, wave, rank, col);
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      if (t0 + k < 0) continue;
      float hb[V], vx[V], vi[V], vr[V];
#pragma unroll
      for (int j = 0; j < V; ++j) hb[j] = Quad<T>::get(rh[k], j);
      if (t0 + k == 0) load_state(a.s_first, a, p, hb);
      grads_of<T>(slope, fe[k], fa[k], rg[k], ri[k], rx[k], hb, at, sum, vx, vi, vr);
      if (p.on) {
        Quad<T>::put(ox.at(ts, k), vx);
        Quad<T>::put(oi.at(ts, k), vi);
        Quad<T>::put(orr.at(ts, k), vr);
      }
    }
    if (last && a.s_out && wave == 0) a.s_out[state_at] = out;
  } else if (n == 0 && a.s_out && wave == 0) {
    a.s_out[state_at] = a.s_in ? a.s_in[state_at] : 0.f;
  }
  zero_stretch<T, kTile>(a, a.dx, p, len, (int)n, run);
  zero_stretch<T, kTile>(a, a.di, p, len, (int)n, run);
  zero_stretch<T, kTile>(a, a.dr, p, len, (int)n, run);
  if (a.part) {
    __shared__ __align__(16) float all[kRuns * kSlab];
    block_sums(a, sum, all, wave * TW + rank, col, slab, p.b * q.tiles + n);
  }
}

// The words before a launch, and its ticket.
__global__ void __launch_bounds__(256) k_recur_clear(uint4* __restrict__ p, int64_t n, uint32_t* __restrict__ ticket) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = uint4{kNone, kNone, kNone, kNone};
  if (i == 0) *ticket = 0;
}

// ddecay from the blocks' sums: 16 channels a block, 64 threads a channel (every
// 64th partial row in order, then the 64 sums in order).
__global__ void __launch_bounds__(1024)
    k_recur_ddecay(const float* __restrict__ part, int64_t rows, int32_t width, const float* __restrict__ decay, float rate,
                   float* __restrict__ ddecay, int32_t accumulate) {
  __shared__ float sh[64][17];
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4, c = blockIdx.x * 16 + cx;
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (int64_t r = ry; r < rows; r += 64) s += part[r * width + c];
  }
  sh[ry][cx] = s;
  __syncthreads();
  if (ry == 0 && c < width) {
#pragma unroll
    for (int q = 1; q < 64; ++q) s += sh[q][cx];
    s *= -rate / (1.f + expf(-decay[c]));
    ddecay[c] = accumulate ? ddecay[c] + s : s;
  }
}

template <class T>
__global__ void __launch_bounds__(256)
    k_recur_step(const RecurArgs a, float* __restrict__ states, const int32_t* __restrict__ slots, int64_t n_slots) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t b = id / a.width;
  const int c = (int)(id - b * a.width);
  if (b >= a.batch) return;
  const int64_t slot = slots ? slots[b] : b;
  float h = 0.f;
  if (slot >= 0 && slot < n_slots) {
    auto get = [&](const Rows& x) { return Elt<T>::get(static_cast<const T*>(x.p) + b * x.sb + c); };
    float* st = states + slot * a.width + c;
    const float l = -slope_of(a.decay[c], a.rate) * sigm(get(a.r)), f = __builtin_amdgcn_exp2f(l);
    h = fmaf(f, *st, __builtin_amdgcn_sqrtf(rest_of(l, f)) * sigm(get(a.i)) * get(a.x));
    *st = h;
  }
  T* o = static_cast<T*>(a.h.p) + b * a.h.sb + c;
  if constexpr (sizeof(T) == 4) {
    *o = h;
  } else {
    *o = f2bf(h);
  }
}

// ---- host ---------------------------------------------------------------------------
constexpr int64_t kMaxToken = (int64_t)1 << 21;  // (a tile has at most 2^8 tokens of 4-byte values)
// Tokens of a thread's run: fewer registers and more waves against the shuffles and LDS
// of a tile.  Where a block walks a sequence, bfloat16: backward of 64 x 512 tokens of
// 2048 channels 251 us with 2, 257 with 1, 248 with 4, of 2048 x 96 tokens of 64 channels
// 54, 52 and 62; forward of the former 119 with 4, 117 with 2, 127 with 8, of 2048 x 1024
// tokens of 64 channels 217, 222 and 224.  A wave for each of 8192 float32 histories of 24
// tokens, backward: 62 us with 1, 67 with 2.
constexpr int fwd_run(bool wave) { return wave ? 2 : 4; }
constexpr int bwd_run(bool wave) { return wave ? 1 : 2; }
// In a chain the whole tile is in flight at once: one history of 65521 tokens of 1024
// channels, bfloat16, 132 us with 14, 137 with 10 or 12, 142 with 16; 8 x 2048 tokens of
// 1024 channels, float32, 64 us with 8, 67 with 10, 69 with 6, their backward 128 us with
// 5, 127 with 4 or 6; ragged in bfloat16, 2048 channels, 108 us with 9, 110 with 8, 136
// with 10.
constexpr int chain_run(bool bwd, bool f32) { return bwd ? (f32 ? 5 : 9) : (f32 ? 8 : 14); }

struct Split {
  bool wave;         // a wave for each sequence
  bool chain;        // a block for each tile, in one pass
  int32_t slabs, tiles;
  int64_t rows;      // blocks of a slab
  int32_t stride;    // WAVE backward: sequences between two of one wave
};

Split split_of(const hg_recur_desc* A, bool bwd) {
  Split s{};
  s.slabs = (int32_t)cdiv(A->width, kSlab);
  const int64_t pairs = (int64_t)A->batch * s.slabs;
  // Up to a tile of 64 tokens, a wave each (8192 histories of 64 bfloat16 channels: of 24
  // tokens forward 23 us, 61 in blocks, backward 57, 86; of 64 tokens 55, 65 and 123, 140; of
  // 128 tokens 116, 113 and 230, 236).
  s.wave = A->t <= 64;
  if (s.wave) {
    s.rows = cdiv(A->batch, kNW);
    if (bwd) s.rows = std::min<int64_t>(s.rows, std::max<int64_t>(1, cdiv(2048, s.slabs)));
    s.stride = (int32_t)(s.rows * kNW);
    return s;
  }
  // Few sequences, up to three blocks for two CUs: one pass, a block a tile (64 bfloat16
  // channels, 256 of 4096 tokens: forward 129 us, 137 where a block walks each, backward 287,
  // 346; 384 of 2048: 104, 99 and 227, 224; 512 of 2048: 132, 115 and 289, 232).  Walked in
  // segments by a block each, after a pass that composes the segments' steps, the long history
  // above took 219 us.
  const int64_t tile = (int64_t)kNW * TW * chain_run(bwd, A->dtype == HG_DTYPE_F32);
  s.chain = pairs < 384 && pairs * cdiv(A->t, tile) < (int64_t)1 << 24;  // (a grid has fewer than 2^32 threads)
  s.tiles = s.chain ? (int32_t)cdiv(A->t, tile) : 1;
  s.rows = (int64_t)A->batch * s.tiles;
  return s;
}

struct Bufs {
  float* part = nullptr;
  uint32_t* words = nullptr;  // a chain's steps, then its values, then the ticket
  int64_t clear = 0;          // of them before the ticket
};
int64_t chain_groups(const Split& s) { return cdiv(s.tiles, kGroup); }
template <class Mem>
Bufs take(const hg_recur_desc* A, bool bwd, Mem& m) {
  const Split s = split_of(A, bwd);
  const int64_t pairs = (int64_t)A->batch * s.slabs;
  Bufs b;
  b.part = m.template take<float>(bwd ? s.rows * A->width : 0);
  if (s.chain) {
    b.clear = pairs * (2 * s.tiles + chain_groups(s)) * kSlab;
    b.words = m.template take<uint32_t>(b.clear + 4);
  }
  return b;
}

int check(const hg_recur_desc* A, const char* what) {
  if (!A) return fail(HG_ERR_ARG, "%s: null descriptor", what);
  if (A->t < 0 || A->batch < 0 || A->width < 1 || !(A->rate > 0.f) || !std::isfinite(A->rate))
    return fail(HG_ERR_ARG, "%s: batch=%d t=%lld width=%d rate=%g", what, A->batch, (long long)A->t, A->width, (double)A->rate);
  if (A->dtype != HG_DTYPE_F32 && A->dtype != HG_DTYPE_BF16) return fail(HG_ERR_ARG, "%s: dtype %d", what, A->dtype);
  if (A->width < V) return fail(HG_ERR_UNSUPPORTED, "%s: width %d is below %d", what, A->width, V);
  // (a grid has fewer than 2^32 threads: 256 for each slab of a sequence)
  if (A->width > 1 << 20 || A->t > (int64_t)1 << 40 || (int64_t)A->batch * cdiv(A->width, kSlab) >= (int64_t)1 << 22 ||
      (int64_t)A->batch * A->width >= ((int64_t)1 << 32) - 256)
    return fail(HG_ERR_UNSUPPORTED, "%s: %d sequences of %lld tokens and %d channels are too many", what, A->batch,
                (long long)A->t, A->width);
  return HG_OK;
}

// The rows of a call; a single token's stride is never walked.
int rows_in(const hg_recur_desc* A, const char* what, const hg_heads* x, const char* name, bool out, Rows* r) {
  HG_TRY(check_rows(what, x, name, out, A->batch, A->t, A->width, A->dtype));
  if (A->t > 1 && x->token > kMaxToken)
    return fail(HG_ERR_UNSUPPORTED, "%s: tokens of %s are %lld apart", what, name, (long long)x->token);
  *r = Rows{x->p, x->batch, A->t > 1 ? x->token : 0};
  return HG_OK;
}

RecurArgs args_of(const hg_recur_desc* A, const Split& s, const float* decay, const int32_t* lens) {
  RecurArgs a{};
  a.decay = decay;
  a.lens = lens;
  a.t = A->t;
  a.batch = A->batch;
  a.width = A->width;
  a.slabs = s.slabs;
  a.rate = A->rate;
  return a;
}

// A chain's words set, and where they are.
int clear_chain(const RecurArgs& a, const Split& s, const Bufs& b, Chain* q, hipStream_t st) {
  const int64_t pairs = (int64_t)a.batch * a.slabs;
  q->step = reinterpret_cast<uint64_t*>(b.words);
  q->value = b.words + pairs * 2 * s.tiles * kSlab;
  q->ticket = b.words + b.clear;
  q->tiles = s.tiles;
  q->groups = (int32_t)chain_groups(s);
  q->pairs = (uint32_t)pairs;
  HG_LAUNCH("recur_clear", k_recur_clear, dim3((unsigned)cdiv(b.clear / 4, 256)), dim3(256), 0, st, reinterpret_cast<uint4*>(b.words),
            b.clear / 4, q->ticket);
  return HG_OK;
}

template <class T>
int launch_fwd(const RecurArgs& a, const Split& s, const Bufs& b, hipStream_t st) {
  if (s.chain) {
    Chain q{};
    HG_TRY(clear_chain(a, s, b, &q, st));
    HG_LAUNCH("recur_chain", (k_recur_chain_fwd<T, chain_run(false, sizeof(T) == 4)>), dim3((unsigned)(s.rows * s.slabs)),
              dim3(kNW * 64), 0, st, a, q);
    return HG_OK;
  }
  const dim3 grid((unsigned)(s.rows * s.slabs)), block(kNW * 64);
  if (s.wave) {
    HG_LAUNCH("recur", (k_recur_fwd<T, fwd_run(true), true>), grid, block, 0, st, a);
  } else {
    HG_LAUNCH("recur", (k_recur_fwd<T, fwd_run(false), false>), grid, block, 0, st, a);
  }
  return HG_OK;
}

template <class T>
int launch_bwd(const RecurArgs& a, const Split& s, const Bufs& b, hipStream_t st) {
  if (s.chain) {
    Chain q{};
    HG_TRY(clear_chain(a, s, b, &q, st));
    HG_LAUNCH("recur_bwd_chain", (k_recur_chain_bwd<T, chain_run(true, sizeof(T) == 4)>), dim3((unsigned)(s.rows * s.slabs)),
              dim3(kNW * 64), 0, st, a, q);
    return HG_OK;
  }
  const dim3 grid((unsigned)(s.rows * s.slabs)), block(kNW * 64);
  if (s.wave) {
    HG_LAUNCH("recur_bwd", (k_recur_bwd<T, bwd_run(true), true>), grid, block, 0, st, a, s.stride);
  } else {
    HG_LAUNCH("recur_bwd", (k_recur_bwd<T, bwd_run(false), false>), grid, block, 0, st, a, 1);
  }
  return HG_OK;
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" size_t hg_recur_fwd_workspace_size(const hg_recur_desc* A) {
  if (check(A, "workspace size") != HG_OK) return 0;
  Sizer m;
  take(A, false, m);
  return m.used;
}

extern "C" size_t hg_recur_bwd_workspace_size(const hg_recur_desc* A) {
  if (check(A, "workspace size") != HG_OK) return 0;
  Sizer m;
  take(A, true, m);
  return m.used;
}

extern "C" int hg_recur_fwd(const hg_recur_desc* A, const hg_heads* x, const hg_heads* r, const hg_heads* i,
                            const float* decay, const int32_t* lens, const float* state, const hg_heads* h,
                            float* state_out, void* ws, size_t ws_bytes, void* stream) {
  const char* what = "hg_recur_fwd";
  HG_TRY(check(A, what));
  Rows rx, rr, ri, rh;
  HG_TRY(rows_in(A, what, x, "x", false, &rx));
  HG_TRY(rows_in(A, what, r, "r", false, &rr));
  HG_TRY(rows_in(A, what, i, "i", false, &ri));
  HG_TRY(rows_in(A, what, h, "h", true, &rh));
  if (A->batch == 0) return HG_OK;
  if (!decay) return fail(HG_ERR_ARG, "%s: null decay", what);
  for (const hg_heads* v : {x, r, i})
    if (rows_meet(h, v, A->batch, A->t, A->width, A->dtype)) return fail(HG_ERR_ARG, "%s: h overlaps an input", what);
  const size_t states = (size_t)A->batch * A->width * 4;
  if (ranges_meet(state, states, state_out, states)) return fail(HG_ERR_ARG, "%s: state_out overlaps state", what);
  Sizer need;
  take(A, false, need);
  HG_TRY(check_workspace(what, ws, ws_bytes, need.used));
  Arena m(ws, ws_bytes);
  const Split s = split_of(A, false);
  RecurArgs a = args_of(A, s, decay, lens);
  const Bufs b = take(A, false, m);
  a.x = rx;
  a.r = rr;
  a.i = ri;
  a.h = rh;
  a.s_in = state;
  a.s_out = state_out;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return A->dtype == HG_DTYPE_F32 ? launch_fwd<float>(a, s, b, st) : launch_fwd<bf16_t>(a, s, b, st);
}

extern "C" int hg_recur_bwd(const hg_recur_desc* A, const hg_heads* x, const hg_heads* r, const hg_heads* i,
                            const float* decay, const int32_t* lens, const float* state, const hg_heads* h,
                            const hg_heads* dh, const float* dstate_out, const hg_heads* dx, const hg_heads* dr,
                            const hg_heads* di, float* ddecay, float* dstate, int32_t accumulate, void* ws,
                            size_t ws_bytes, void* stream) {
  const char* what = "hg_recur_bwd";
  HG_TRY(check(A, what));
  if (accumulate != 0 && accumulate != 1) return fail(HG_ERR_ARG, "%s: accumulate %d", what, accumulate);
  const hg_heads* all[8] = {x, r, i, h, dh, dx, dr, di};
  const char* names[8] = {"x", "r", "i", "h", "dh", "dx", "dr", "di"};
  Rows in[8];
  for (int k = 0; k < 8; ++k) HG_TRY(rows_in(A, what, all[k], names[k], k >= 5, &in[k]));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (A->batch == 0) return ddecay && !accumulate ? fill_f32(ddecay, 0.f, A->width, st) : HG_OK;
  if (!decay) return fail(HG_ERR_ARG, "%s: null decay", what);
  for (int k = 5; k < 8; ++k)
    for (int q = 0; q < k; ++q)
      if (rows_meet(all[k], all[q], A->batch, A->t, A->width, A->dtype))
        return fail(HG_ERR_ARG, "%s: %s overlaps %s", what, names[k], names[q]);
  const size_t states = (size_t)A->batch * A->width * 4, vec = (size_t)A->width * 4;
  if (ranges_meet(dstate, states, state, states) || ranges_meet(dstate, states, dstate_out, states))
    return fail(HG_ERR_ARG, "%s: dstate overlaps an input", what);
  if (ranges_meet(ddecay, vec, decay, vec)) return fail(HG_ERR_ARG, "%s: ddecay overlaps decay", what);
  Sizer need;
  take(A, true, need);
  HG_TRY(check_workspace(what, ws, ws_bytes, need.used));
  Arena m(ws, ws_bytes);
  const Split s = split_of(A, true);
  const Bufs b = take(A, true, m);
  RecurArgs a = args_of(A, s, decay, lens);
  a.part = ddecay ? b.part : nullptr;
  a.x = in[0];
  a.r = in[1];
  a.i = in[2];
  a.h = in[3];
  a.dh = in[4];
  a.dx = in[5];
  a.dr = in[6];
  a.di = in[7];
  a.s_first = state;
  a.s_in = dstate_out;
  a.s_out = dstate;
  HG_TRY(A->dtype == HG_DTYPE_F32 ? launch_bwd<float>(a, s, b, st) : launch_bwd<bf16_t>(a, s, b, st));
  if (ddecay)
    HG_LAUNCH("recur_ddecay", k_recur_ddecay, dim3((unsigned)cdiv(A->width, 16)), dim3(1024), 0, st, a.part, s.rows, A->width,
              decay, A->rate, ddecay, accumulate);
  return HG_OK;
}

extern "C" int hg_recur_step(const hg_recur_desc* A, const hg_heads* x, const hg_heads* r, const hg_heads* i,
                             const float* decay, float* states, const int32_t* slots, int64_t n_slots,
                             const hg_heads* h, void* stream) {
  const char* what = "hg_recur_step";
  HG_TRY(check(A, what));
  if (A->t != 1) return fail(HG_ERR_ARG, "%s: t=%lld, one token a row", what, (long long)A->t);
  Rows rx, rr, ri, rh;
  HG_TRY(rows_in(A, what, x, "x", false, &rx));
  HG_TRY(rows_in(A, what, r, "r", false, &rr));
  HG_TRY(rows_in(A, what, i, "i", false, &ri));
  HG_TRY(rows_in(A, what, h, "h", true, &rh));
  if (n_slots < 0 || (!slots && n_slots < A->batch))
    return fail(HG_ERR_ARG, "%s: %lld states for %d rows", what, (long long)n_slots, A->batch);
  if (A->batch == 0) return HG_OK;
  if (!decay || (!states && n_slots > 0)) return fail(HG_ERR_ARG, "%s: null pointer", what);
  for (const hg_heads* v : {x, r, i})
    if (rows_meet(h, v, A->batch, 1, A->width, A->dtype)) return fail(HG_ERR_ARG, "%s: h overlaps an input", what);
  RecurArgs a{};
  a.decay = decay;
  a.batch = A->batch;
  a.width = A->width;
  a.rate = A->rate;
  a.x = rx;
  a.r = rr;
  a.i = ri;
  a.h = rh;
  const dim3 grid((unsigned)cdiv((int64_t)A->batch * A->width, 256));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (A->dtype == HG_DTYPE_F32) {
    HG_LAUNCH("recur_step", k_recur_step<float>, grid, dim3(256), 0, st, a, states, slots, n_slots);
  } else {
    HG_LAUNCH("recur_step", k_recur_step<bf16_t>, grid, dim3(256), 0, st, a, states, slots, n_slots);
  }
  return HG_OK;
}
