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
// again from the value that reaches it.  So a block takes 4 NW K tokens of 64
// channels at a time with one barrier, every value is read and written once, and
// what is serial is a sequence's tiles.  One wave does so alone where sequences
// are many (WAVE: no barrier).  Where there are few, the history is cut into
// segments: a first pass composes each segment's step (k_recur_sums), and the
// segments' blocks start from the steps before theirs.
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
  float* sums;           // [batch][segs][2][width] steps of the segments
  float* part;           // [blocks of a slab][width] sums of dlog sigmoid(r), or null
  int64_t t, seg_len;
  int32_t batch, width, slabs, segs;
  float rate;
};

template <class T>
using Quad = Vec<T, V>;

__device__ __forceinline__ float sigm(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z)); }

// rate softplus(decay) log2 e: the factor is 2^(-that sigmoid(r))
__device__ __forceinline__ float slope_of(float decay, float rate) {
  return rate * kLog2e * (fmaxf(decay, 0.f) + log1pf(expf(-fabsf(decay))));
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
  int64_t b, t_beg, t_end, out_end;  // tokens of the segment: inside the sequence, and with the rows past it
  int32_t seg, c0;                   // first channel of the thread
  bool on;                           // no thread before has the same channels
};
__device__ __forceinline__ int64_t len_of(const RecurArgs& a, int64_t b) {
  if (!a.lens) return a.t;
  const int32_t n = a.lens[b];
  return n < 0 ? 0 : (n < a.t ? n : a.t);
}
template <bool WAVE>
__device__ __forceinline__ Place place_of(const RecurArgs& a, int wave, int col) {
  Place p;
  const uint32_t id = blockIdx.x, rest = id / (uint32_t)a.slabs, slab = id - rest * (uint32_t)a.slabs;
  if constexpr (WAVE) {
    p.b = (int64_t)rest * kNW + wave;
    p.seg = 0;
  } else {
    p.b = rest / (uint32_t)a.segs;
    p.seg = (int32_t)(rest - (uint32_t)p.b * (uint32_t)a.segs);
  }
  const int c = (int)slab * kSlab + col * V;
  p.on = c < a.width;
  p.c0 = c < a.width - V ? c : a.width - V;
  const int64_t len = p.b < a.batch ? len_of(a, p.b) : 0;
  p.t_beg = p.seg * a.seg_len;
  p.out_end = p.t_beg + a.seg_len < a.t ? p.t_beg + a.seg_len : a.t;
  p.t_end = len < p.out_end ? len : p.out_end;
  if (p.t_end < p.t_beg) p.t_end = p.t_beg;
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

// The steps of the segments [from, to) in their order, on y.
__device__ __forceinline__ void run_segments(const RecurArgs& a, const Place& p, int from, int to, int dir, float (&y)[V]) {
  const float* s = a.sums + p.b * a.segs * 2 * (int64_t)a.width + p.c0;
  for (int q = from; q != to; q += dir) {
    const float* f = s + q * 2 * (int64_t)a.width;
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = fmaf(f[j], y[j], f[a.width + j]);
  }
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
  if (!WAVE && p.seg) run_segments(a, p, 0, p.seg, 1, y);
  const Stream<T> sx(a.x, p, run * K), sr(a.r, p, run * K), si(a.i, p, run * K), sh(a.h, p, run * K);
  typename Quad<T>::raw rx[K] = {}, rr[K] = {}, ri[K] = {};
  auto fetch = [&](auto full, int64_t ts) {
    constexpr bool FULL = decltype(full)::value;
    load<T, K, FULL>(rr, sr, ts, ts + run * K, p.t_beg, p.t_end);
    load<T, K, FULL>(ri, si, ts, ts + run * K, p.t_beg, p.t_end);
    load<T, K, FULL>(rx, sx, ts, ts + run * K, p.t_beg, p.t_end);
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
  int64_t ts = p.t_beg;
  if (ts + kTile <= p.t_end) {
    fetch(Bool<true>{}, ts);
  } else {
    fetch(Bool<false>{}, ts);
  }
  for (; ts + kTile <= p.t_end; ts += kTile) tile(Bool<true>{}, ts);
  if (ts < p.t_end) tile(Bool<false>{}, ts);
  zero_rows<T>(a.h, p, run, WAVE ? TW : kNW * TW);
  if (a.s_out && p.on && run == 0 && p.seg == a.segs - 1) {
#pragma unroll
    for (int j = 0; j < V; ++j) a.s_out[p.b * a.width + p.c0 + j] = y[j];
  }
}

// The step of each segment.  A thread takes one run of the segment's tokens and
// walks it K at a time; the block composes the runs at the end.  BACK: the
// backward's, from the last token.
template <class T, int K, bool BACK>
__global__ void __launch_bounds__(kNW * 64) k_recur_sums(const RecurArgs a) {
  __shared__ __align__(16) float lds[kNW * 2 * kSlab];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane % CL, rank = lane / CL;
  const Place p = place_of<false>(a, wave, col);
  // (the steps of the last segment of a walk lead nowhere)
  if (p.seg == (BACK ? 0 : a.segs - 1)) return;
  // run q of the segment in the walk's order: tokens [beg + q per, ..) forward, backward down from end - q per
  const int q = wave * TW + rank;
  const int64_t n = p.t_end - p.t_beg, per = ((n + kNW * TW - 1) / (kNW * TW) + K - 1) / K * K;
  const int64_t first = BACK ? p.t_end - kNW * TW * per : p.t_beg;  // (may be before the segment)
  const int64_t skip = (BACK ? kNW * TW - 1 - q : q) * per;
  const Stream<T, int64_t> sx(BACK ? a.dh : a.x, p, skip), sr(a.r, p, skip), si(a.i, p, skip);
  float slope[V];
  Step s;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    slope[j] = -slope_of(a.decay[p.c0 + j], a.rate);
    s.a[j] = 1.f;
    s.b[j] = 0.f;
  }
  typename Quad<T>::raw rx[K] = {}, rr[K] = {}, ri[K] = {};
  auto fetch = [&](auto full, int64_t ts) {
    constexpr bool FULL = decltype(full)::value;
    load<T, K, FULL>(rr, sr, ts, ts + skip, p.t_beg, p.t_end);
    if constexpr (!BACK) load<T, K, FULL>(ri, si, ts, ts + skip, p.t_beg, p.t_end);
    load<T, K, FULL>(rx, sx, ts, ts + skip, p.t_beg, p.t_end);
  };
  // whether all runs' tokens of a round lie inside: only the last run forward, backward the first, may not
  const bool whole = per * kNW * TW == n;
  const auto walk = [&](auto full) {
    constexpr bool FULL = decltype(full)::value;
    const int64_t step = BACK ? -K : K;
    int64_t ts = BACK ? first + per - K : first;
    if (per > 0) fetch(full, ts);
    for (int64_t i = 0; i < per; i += K, ts += step) {
      float fa[K][V], fu[K][V];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int64_t t = ts + skip + k;
        const bool in = FULL || (t >= p.t_beg && t < p.t_end);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float l = slope[j] * sigm(Quad<T>::get(rr[k], j));
          const float f = __builtin_amdgcn_exp2f(l);
          float u = Quad<T>::get(rx[k], j);
          if constexpr (BACK) {
            u *= f;
          } else {
            u *= __builtin_amdgcn_sqrtf(rest_of(l, f)) * sigm(Quad<T>::get(ri[k], j));
          }
          fa[k][j] = in ? f : 1.f;
          fu[k][j] = in ? u : 0.f;
        }
      }
      if (i + K < per) fetch(full, ts + step);
#pragma unroll
      for (int o = 0; o < K; ++o) {
        const int k = BACK ? K - 1 - o : o;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          s.a[j] *= fa[k][j];
          s.b[j] = fmaf(fa[k][j], s.b[j], fu[k][j]);
        }
      }
    }
  };
  if (whole) {
    walk(Bool<true>{});
  } else {
    walk(Bool<false>{});
  }
  // the whole segment's step: the value that leaves it from 0, and the product of its factors
  Step before;
  compose_wave(s, before, rank);
  if (rank == TW - 1) {
    *reinterpret_cast<f32x4*>(lds + wave * 2 * kSlab + col * V) = f32x4{s.a[0], s.a[1], s.a[2], s.a[3]};
    *reinterpret_cast<f32x4*>(lds + wave * 2 * kSlab + kSlab + col * V) = f32x4{s.b[0], s.b[1], s.b[2], s.b[3]};
  }
  __syncthreads();
  if (q == 0 && p.on) {
    f32x4 ya = f32x4{1.f, 1.f, 1.f, 1.f}, yb = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kNW; ++w) {
      const f32x4 qa = *reinterpret_cast<const f32x4*>(lds + w * 2 * kSlab + col * V);
      const f32x4 qb = *reinterpret_cast<const f32x4*>(lds + w * 2 * kSlab + kSlab + col * V);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        yb[j] = fmaf(qa[j], yb[j], qb[j]);
        ya[j] *= qa[j];
      }
    }
    float* o = a.sums + (p.b * a.segs + p.seg) * 2 * (int64_t)a.width + p.c0;
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = ya[j], o[a.width + j] = yb[j];
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
    if (!WAVE && p.seg < a.segs - 1) run_segments(a, p, a.segs - 1, p.seg, -1, y);
    const Stream<T> sx(a.x, p, skip), sr(a.r, p, skip), si(a.i, p, skip), sh(a.h, p, skip), sg(a.dh, p, skip), ox(a.dx, p, skip),
        orr(a.dr, p, skip), oi(a.di, p, skip);
    typename Quad<T>::raw rx[K] = {}, rr[K] = {}, ri[K] = {}, rh[K] = {}, rg[K] = {};
    // the tile of tokens ts .. ts + kTile - 1 (row k of rh: h before the thread's token k); FULL: it begins after t_beg
    auto fetch = [&](auto full, int64_t ts) {
      constexpr bool FULL = decltype(full)::value;
      load<T, K, FULL>(rr, sr, ts, ts + skip, p.t_beg, p.t_end);
      load<T, K, FULL>(rg, sg, ts, ts + skip, p.t_beg, p.t_end);
      load<T, K, FULL>(ri, si, ts, ts + skip, p.t_beg, p.t_end);
      load<T, K, FULL>(rx, sx, ts, ts + skip, p.t_beg, p.t_end);
      load<T, K, FULL>(rh, sh, ts - 1, ts - 1 + skip, p.t_beg ? p.t_beg - 1 : 0, p.t_end);
    };
    int odd = 0;
    auto tile = [&](auto full, int64_t ts) {
      constexpr bool FULL = decltype(full)::value;
      const int64_t t0 = ts + skip;
      float fs[K][V], fa[K][V], gh[K][V];
      Step s;
#pragma unroll
      for (int j = 0; j < V; ++j) s.a[j] = 1.f, s.b[j] = 0.f;
#pragma unroll
      for (int k = K - 1; k >= 0; --k) {
        const bool in = FULL || t0 + k >= p.t_beg;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          fs[k][j] = sigm(Quad<T>::get(rr[k], j));
          const float f = __builtin_amdgcn_exp2f(slope[j] * fs[k][j]);
          fa[k][j] = in ? f : 1.f;
          gh[k][j] = in ? Quad<T>::get(rg[k], j) : 0.f;
          s.b[j] = fa[k][j] * (s.b[j] + gh[k][j]);
          s.a[j] *= fa[k][j];
        }
      }
      float at[V];
      compose<WAVE>(s, y, at, lds + (WAVE ? 0 : odd * kNW * 2 * kSlab), wave, rank, col);
      odd ^= 1;
#pragma unroll
      for (int k = K - 1; k >= 0; --k) {
        if (!FULL && t0 + k < p.t_beg) continue;
        float hb[V], vx[V], vi[V], vr[V];
#pragma unroll
        for (int j = 0; j < V; ++j) hb[j] = Quad<T>::get(rh[k], j);
        if (!FULL && t0 + k == 0) load_state(a.s_first, a, p, hb);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float f = fa[k][j], l = slope[j] * fs[k][j], g = gh[k][j] + at[j];
          at[j] = f * g;
          // (1 - a^2 at least 2^-120, below which l = 0, so that its root's inverse is finite)
          const float m = rest_of(l, f), iq = __builtin_amdgcn_rsqf(fmaxf(m, 7.5e-37f)), q = m * iq;
          const float sg1 = sigm(Quad<T>::get(ri[k], j)), x = Quad<T>::get(rx[k], j), gs = g * sg1;
          vx[j] = gs * q;
          vi[j] = vx[j] * x * (1.f - sg1);
          const float dl = f * fmaf(g, hb[j], -gs * x * f * iq);
          sum[j] = fmaf(dl, fs[k][j], sum[j]);
          vr[j] = dl * (l * 0.69314718055994531f) * (1.f - fs[k][j]);
        }
        if (p.on) {
          Quad<T>::put(ox.at(ts, k), vx);
          Quad<T>::put(oi.at(ts, k), vi);
          Quad<T>::put(orr.at(ts, k), vr);
        }
      }
      // the tile before; one that holds token 0 is not full (its h before comes from the state)
      if (ts - kTile > p.t_beg) {
        fetch(Bool<true>{}, ts - kTile);
      } else if (ts > p.t_beg) {
        fetch(Bool<false>{}, ts - kTile);
      }
    };
    int64_t ts = p.t_end - kTile;
    if (ts > p.t_beg) {
      fetch(Bool<true>{}, ts);
    } else {
      fetch(Bool<false>{}, ts);
    }
    for (; ts > p.t_beg; ts -= kTile) tile(Bool<true>{}, ts);
    if (ts + kTile > p.t_beg) tile(Bool<false>{}, ts);
    const int ranks = WAVE ? TW : kNW * TW;
    zero_rows<T>(a.dx, p, run, ranks);
    zero_rows<T>(a.di, p, run, ranks);
    zero_rows<T>(a.dr, p, run, ranks);
    if (a.s_out && p.on && run == 0 && p.seg == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) a.s_out[p.b * a.width + p.c0 + j] = y[j];
    }
    if (!WAVE) break;
  }
  if (!a.part) return;
  // the block's sums of its runs, in order
  __syncthreads();
  float* all = lds;  // [NW * TW][slab]
  static_assert(kNW * TW * kSlab <= 2 * kNW * 2 * kSlab, "the sums fit the block's LDS");
#pragma unroll
  for (int j = 0; j < V; ++j) all[(wave * TW + rank) * kSlab + col * V + j] = sum[j];
  __syncthreads();
  const uint32_t rest = blockIdx.x / (uint32_t)a.slabs, slab = blockIdx.x - rest * (uint32_t)a.slabs;
  for (int c = threadIdx.x; c < kSlab; c += kNW * 64) {
    const int ch = (int)slab * kSlab + c;
    if (ch >= a.width) continue;
    // the thread that has channel ch: the last ones start at width - V
    const int own = c / V, c0 = (int)slab * kSlab + own * V, shift = c0 < a.width - V ? 0 : c0 - (a.width - V);
    float s = 0.f;
    for (int q = 0; q < kNW * TW; ++q) s += all[q * kSlab + c + shift];
    a.part[(int64_t)rest * a.width + ch] = s;
  }
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
// Tokens of a thread's run.  Fewer registers and more waves against the shuffles and
// LDS of a tile: one history of 65521 tokens of 1024 channels, bfloat16, 219 us with 4,
// 236 with 8; backward of 8 x 2048 tokens of 2048 channels 121 us with 2, 127 with 4; a
// wave for each of 8192 histories of 24 tokens, float32, 62 us with 1, 67 with 2.
constexpr int fwd_run(bool wave) { return wave ? 2 : 4; }
constexpr int bwd_run(bool wave) { return wave ? 1 : 2; }

struct Split {
  bool wave;         // a wave for each sequence
  int32_t slabs, segs;
  int64_t seg_len;
  int64_t rows;      // blocks of a slab
  int32_t stride;    // WAVE backward: sequences between two of one wave
};

Split split_of(const hg_recur_desc* A, bool bwd) {
  Split s{};
  s.slabs = (int32_t)cdiv(A->width, kSlab);
  const int64_t pairs = (int64_t)A->batch * s.slabs;
  s.wave = pairs >= 4096 || A->t <= 64;
  s.segs = 1;
  s.seg_len = std::max<int64_t>(A->t, 1);
  if (s.wave) {
    s.rows = cdiv(A->batch, kNW);
    if (bwd) s.rows = std::min<int64_t>(s.rows, std::max<int64_t>(1, cdiv(2048, s.slabs)));
    s.stride = (int32_t)(s.rows * kNW);
    return s;
  }
  const int64_t tile = (int64_t)kNW * TW * (bwd ? bwd_run(false) : fwd_run(false));
  const int64_t n = std::min<int64_t>(1024 / std::max<int64_t>(pairs, 1), A->t / (4 * tile));
  if (n > 1) {
    s.seg_len = cdiv(cdiv(A->t, n), tile) * tile;
    s.segs = (int32_t)cdiv(A->t, s.seg_len);
  }
  s.rows = (int64_t)A->batch * s.segs;
  return s;
}

struct Bufs {
  float *sums = nullptr, *part = nullptr;
};
template <class Mem>
Bufs take(const hg_recur_desc* A, bool bwd, Mem& m) {
  const Split s = split_of(A, bwd);
  Bufs b;
  b.sums = m.template take<float>(s.segs > 1 ? (int64_t)A->batch * s.segs * 2 * A->width : 0);
  b.part = m.template take<float>(bwd ? s.rows * A->width : 0);
  return b;
}

int check(const hg_recur_desc* A, const char* what) {
  if (!A) return fail(HG_ERR_ARG, "%s: null descriptor", what);
  if (A->t < 0 || A->batch < 0 || A->width < 1 || !(A->rate > 0.f) || !std::isfinite(A->rate))
    return fail(HG_ERR_ARG, "%s: batch=%d t=%lld width=%d rate=%g", what, A->batch, (long long)A->t, A->width, (double)A->rate);
  if (A->dtype != HG_DTYPE_F32 && A->dtype != HG_DTYPE_BF16) return fail(HG_ERR_ARG, "%s: dtype %d", what, A->dtype);
  if (A->width < V) return fail(HG_ERR_UNSUPPORTED, "%s: width %d is below %d", what, A->width, V);
  // (a grid has fewer than 2^32 threads: 512 for each slab of a sequence's segment)
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
  a.seg_len = s.seg_len;
  a.batch = A->batch;
  a.width = A->width;
  a.slabs = s.slabs;
  a.segs = s.segs;
  a.rate = A->rate;
  return a;
}

template <class T>
int launch_fwd(const RecurArgs& a, const Split& s, hipStream_t st) {
  const dim3 grid((unsigned)(s.rows * s.slabs)), block(kNW * 64);
  if (s.segs > 1) HG_LAUNCH("recur_sums", (k_recur_sums<T, fwd_run(false), false>), grid, block, 0, st, a);
  if (s.wave) {
    HG_LAUNCH("recur", (k_recur_fwd<T, fwd_run(true), true>), grid, block, 0, st, a);
  } else {
    HG_LAUNCH("recur", (k_recur_fwd<T, fwd_run(false), false>), grid, block, 0, st, a);
  }
  return HG_OK;
}

template <class T>
int launch_bwd(const RecurArgs& a, const Split& s, hipStream_t st) {
  const dim3 grid((unsigned)(s.rows * s.slabs)), block(kNW * 64);
  if (s.segs > 1) HG_LAUNCH("recur_bwd_sums", (k_recur_sums<T, bwd_run(false), true>), grid, block, 0, st, a);
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
  if (state && state == state_out) return fail(HG_ERR_ARG, "%s: state_out is state", what);
  Sizer need;
  take(A, false, need);
  HG_TRY(check_workspace(what, ws, ws_bytes, need.used));
  Arena m(ws, ws_bytes);
  const Split s = split_of(A, false);
  RecurArgs a = args_of(A, s, decay, lens);
  a.sums = take(A, false, m).sums;
  a.x = rx;
  a.r = rr;
  a.i = ri;
  a.h = rh;
  a.s_in = state;
  a.s_out = state_out;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return A->dtype == HG_DTYPE_F32 ? launch_fwd<float>(a, s, st) : launch_fwd<bf16_t>(a, s, st);
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
  if (dstate && (dstate == state || dstate == dstate_out)) return fail(HG_ERR_ARG, "%s: dstate is an input", what);
  if (ddecay && ddecay == decay) return fail(HG_ERR_ARG, "%s: ddecay is decay", what);
  Sizer need;
  take(A, true, need);
  HG_TRY(check_workspace(what, ws, ws_bytes, need.used));
  Arena m(ws, ws_bytes);
  const Split s = split_of(A, true);
  const Bufs b = take(A, true, m);
  RecurArgs a = args_of(A, s, decay, lens);
  a.sums = b.sums;
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
  HG_TRY(A->dtype == HG_DTYPE_F32 ? launch_bwd<float>(a, s, st) : launch_bwd<bf16_t>(a, s, st));
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
