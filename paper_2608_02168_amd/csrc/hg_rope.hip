// Norm of queries and keys for each head with the position rotation in the
// same pass.
//
//   y = x r w,  r = 1 / sqrt(mean(x^2) + eps),  then pairs (i, j) of the first
//   `rot` columns turned by the angle of the token's position:
//   (y_i cos - y_j sin, y_j cos + y_i sin)
// backward, with g the upstream row turned back:
//   dw = sum over rows of g x r,   dx = r (g w - x r mean(g w x r))
//
// One read and one write of every row: bound by HBM (32768 tokens of 40 heads of
// 128, bfloat16: 138 us, 5.0 TB/s; backward of 20011 tokens of 24 heads of 64,
// float32: 76 us, 4.9 TB/s; a large copy reaches 4.9).  A head's row is taken by
// G lanes (a power of two), eight columns a lane, in two groups of four so
// chosen that both columns of every pair are in one lane: columns 4 u .. and
// rot / 2 + 4 u .. for pairs (p, p + rot / 2), columns 8 u .. + 7 for adjacent
// pairs and for the columns that are not turned.  The mean is a reduction over
// the G lanes.  A group takes every S-th head of one token, so the token's
// angles and the weights stay in registers over its heads.
#include <cmath>

#include "hg_mfma.h"

namespace hg {
namespace {

constexpr int kMaxD = 256;
constexpr int kThreads = 256;
constexpr int kBwdBlocks = 1024;  // partial rows of the weight gradients at most

struct Heads {
  void* p;
  int64_t st, sh;
};

struct RopeArgs {
  Heads q, k;        // rows x
  Heads gq, gk;      // upstream rows (backward)
  Heads oq, ok;      // rows written
  const float *wq, *wk;
  const float* table;  // [n_pos][rot]: cosines, then sines
  const int32_t* pos;
  int64_t n, n_pos;
  int32_t hq, hk, d, rot, inter;
  int32_t slots;       // S: groups that share a token's heads
  float eps;
  float* part;         // [blocks][2][d] sums of the weight gradients
};

struct Lane {
  int c0, c1;   // first columns of the two groups
  bool turned;  // the columns are turned
};

__device__ __forceinline__ Lane lane_of(int u, int d, int rot, int inter) {
  Lane l;
  l.turned = 8 * u < rot;
  const bool split = l.turned && !inter;
  l.c0 = split ? 4 * u : 8 * u;
  l.c1 = split ? rot / 2 + 4 * u : 8 * u + 4;
  return l;
}

// Cosines and sines of the lane's four pairs at one position: adjacent pairs
// 4 u .. 4 u + 3, or pairs (4 u + i, rot / 2 + 4 u + i).  Either way pair 4 u + i.
__device__ __forceinline__ void angles(const RopeArgs& a, int64_t t, int u, bool turned, f32x4& cs, f32x4& sn) {
  cs = f32x4{1.f, 1.f, 1.f, 1.f};
  sn = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t p = a.pos[t];
  if (p < 0 || p >= a.n_pos) {
    const float x = __builtin_nanf("");
    cs = f32x4{x, x, x, x};
  } else if (turned) {
    const float* row = a.table + p * a.rot + 4 * u;
    cs = *reinterpret_cast<const f32x4*>(row);
    sn = *reinterpret_cast<const f32x4*>(row + a.rot / 2);
  }
}

// The lane's pairs turned by the angles (sign -1: back).  Columns that are not
// turned have cosine 1 and sine 0, or NaN for a position outside the table.
__device__ __forceinline__ void turn(f32x4& x, f32x4& y, const f32x4& cs, const f32x4& sn, float sign, bool inter) {
  f32x4 a = x, b = y;
  if (inter) {
    a = f32x4{x[0], x[2], y[0], y[2]};
    b = f32x4{x[1], x[3], y[1], y[3]};
  }
  f32x4 u, v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float s = sign * sn[i];
    u[i] = a[i] * cs[i] - b[i] * s;
    v[i] = b[i] * cs[i] + a[i] * s;
  }
  if (inter) {
    x = f32x4{u[0], v[0], u[1], v[1]};
    y = f32x4{u[2], v[2], u[3], v[3]};
  } else {
    x = u;
    y = v;
  }
}

template <class T>
__device__ __forceinline__ void store4(T* p, const f32x4& x) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(p) = x;
  } else {
    *reinterpret_cast<uint2*>(p) = uint2{pack2bf(x[0], x[1]), pack2bf(x[2], x[3])};
  }
}

template <int G>
__device__ __forceinline__ float group_sum(float s) {
#pragma unroll
  for (int o = 1; o < G; o <<= 1) s += __shfl_xor(s, o, 64);
  return s;
}

__device__ __forceinline__ float dot8(const f32x4& a, const f32x4& b, const f32x4& c, const f32x4& d) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) s = fmaf(a[i], b[i], s);
#pragma unroll
  for (int i = 0; i < 4; ++i) s = fmaf(c[i], d[i], s);
  return s;
}

__device__ __forceinline__ f32x4 weight4(const float* w, int c) {
  return w ? *reinterpret_cast<const f32x4*>(w + c) : f32x4{1.f, 1.f, 1.f, 1.f};
}

// UNR heads of a token in flight at a time.
template <class T, int G, int UNR>
__global__ void __launch_bounds__(kThreads) k_qk_norm_rope(const RopeArgs a) {
  const int64_t id = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / G;
  const int u = threadIdx.x % G;
  const int64_t t = id / a.slots;
  if (t >= a.n) return;
  const int slot = (int)(id - t * a.slots), H = a.hq + a.hk;
  const bool in = 8 * u < a.d;
  const Lane l = lane_of(in ? u : 0, a.d, a.rot, a.inter);
  const bool inter = a.inter || !l.turned;
  f32x4 cs, sn;
  angles(a, t, in ? u : 0, l.turned, cs, sn);
  const f32x4 wq0 = weight4(a.wq, l.c0), wq1 = weight4(a.wq, l.c1), wk0 = weight4(a.wk, l.c0), wk1 = weight4(a.wk, l.c1);
  const float inv = 1.f / (float)a.d;
  for (int h0 = slot; h0 < H; h0 += a.slots * UNR) {
    typename Elt<T>::raw4_t r0[UNR], r1[UNR];
#pragma unroll
    for (int i = 0; i < UNR; ++i) {
      const int h = h0 + i * a.slots < H ? h0 + i * a.slots : h0;
      const Heads& x = h < a.hq ? a.q : a.k;
      const T* p = static_cast<const T*>(x.p) + t * x.st + (h < a.hq ? h : h - a.hq) * x.sh;
      r0[i] = Elt<T>::raw4(p + l.c0);
      r1[i] = Elt<T>::raw4(p + l.c1);
    }
#pragma unroll
    for (int i = 0; i < UNR; ++i) {
      const int h = h0 + i * a.slots;
      const bool is_q = h < a.hq;
      f32x4 x = Elt<T>::cook4(r0[i]), y = Elt<T>::cook4(r1[i]);
      const float ss = group_sum<G>(in ? dot8(x, x, y, y) : 0.f);
      const float r = 1.f / sqrtf(ss * inv + a.eps);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        x[v] = x[v] * r * (is_q ? wq0[v] : wk0[v]);
        y[v] = y[v] * r * (is_q ? wq1[v] : wk1[v]);
      }
      turn(x, y, cs, sn, 1.f, inter);
      if (in && h < H) {
        const Heads& o = is_q ? a.oq : a.ok;
        T* p = static_cast<T*>(o.p) + t * o.st + (is_q ? h : h - a.hq) * o.sh;
        store4<T>(p + l.c0, x);
        store4<T>(p + l.c1, y);
      }
    }
  }
}

template <class T, int G, int UNR>
__global__ void __launch_bounds__(kThreads) k_qk_norm_rope_bwd(const RopeArgs a) {
  __shared__ float sh[kThreads / G][2][8 * G];
  const int u = threadIdx.x % G, grp = threadIdx.x / G, H = a.hq + a.hk;
  const bool in = 8 * u < a.d;
  const Lane l = lane_of(in ? u : 0, a.d, a.rot, a.inter);
  const bool inter = a.inter || !l.turned;
  const f32x4 wq0 = weight4(a.wq, l.c0), wq1 = weight4(a.wq, l.c1), wk0 = weight4(a.wk, l.c0), wk1 = weight4(a.wk, l.c1);
  const float inv = 1.f / (float)a.d;
  f32x4 dw[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i) dw[i >> 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t groups = (int64_t)gridDim.x * (kThreads / G), items = a.n * a.slots;
  for (int64_t id = (int64_t)blockIdx.x * (kThreads / G) + grp; id < items; id += groups) {
    const int64_t t = id / a.slots;
    const int slot = (int)(id - t * a.slots);
    f32x4 cs, sn;
    angles(a, t, in ? u : 0, l.turned, cs, sn);
    for (int h0 = slot; h0 < H; h0 += a.slots * UNR) {
      typename Elt<T>::raw4_t r0[UNR], r1[UNR], g0[UNR], g1[UNR];
#pragma unroll
      for (int i = 0; i < UNR; ++i) {
        const int h = h0 + i * a.slots < H ? h0 + i * a.slots : h0;
        const bool is_q = h < a.hq;
        const int hh = is_q ? h : h - a.hq;
        const Heads &x = is_q ? a.q : a.k, &g = is_q ? a.gq : a.gk;
        const T *p = static_cast<const T*>(x.p) + t * x.st + hh * x.sh, *gp = static_cast<const T*>(g.p) + t * g.st + hh * g.sh;
        r0[i] = Elt<T>::raw4(p + l.c0);
        r1[i] = Elt<T>::raw4(p + l.c1);
        g0[i] = Elt<T>::raw4(gp + l.c0);
        g1[i] = Elt<T>::raw4(gp + l.c1);
      }
#pragma unroll
      for (int i = 0; i < UNR; ++i) {
        const int h = h0 + i * a.slots;
        if (h >= H) continue;  // the same for the whole group
        const bool is_q = h < a.hq;
        f32x4 x = Elt<T>::cook4(r0[i]), y = Elt<T>::cook4(r1[i]), g = Elt<T>::cook4(g0[i]), e = Elt<T>::cook4(g1[i]);
        turn(g, e, cs, sn, -1.f, inter);
        const float ss = group_sum<G>(in ? dot8(x, x, y, y) : 0.f);
        const float r = 1.f / sqrtf(ss * inv + a.eps);
        f32x4 &d0 = dw[0][0], &d1 = dw[0][1], &e0 = dw[1][0], &e1 = dw[1][1];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          x[v] *= r;
          y[v] *= r;
          const float p = g[v] * x[v], q = e[v] * y[v];
          d0[v] += is_q ? p : 0.f;
          d1[v] += is_q ? q : 0.f;
          e0[v] += is_q ? 0.f : p;
          e1[v] += is_q ? 0.f : q;
          g[v] *= is_q ? wq0[v] : wk0[v];
          e[v] *= is_q ? wq1[v] : wk1[v];
        }
        const float m = group_sum<G>(in ? dot8(g, x, e, y) : 0.f) * inv;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          x[v] = r * (g[v] - x[v] * m);
          y[v] = r * (e[v] - y[v] * m);
        }
        if (in) {
          const Heads& o = is_q ? a.oq : a.ok;
          T* p = static_cast<T*>(o.p) + t * o.st + (is_q ? h : h - a.hq) * o.sh;
          store4<T>(p + l.c0, x);
          store4<T>(p + l.c1, y);
        }
      }
    }
  }
  if (!a.part) return;
  // the block's sums, its groups in order
  if (in) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        sh[grp][k][l.c0 + v] = dw[k][0][v];
        sh[grp][k][l.c1 + v] = dw[k][1][v];
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.d; i += kThreads) {
    const int k = i >= a.d, c = i - k * a.d;
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < kThreads / G; ++q) s += sh[q][k][c];
    a.part[(int64_t)blockIdx.x * 2 * a.d + i] = s;
  }
}

// Weight gradients from the blocks' sums: 16 columns a block, 64 threads a column
// (every 64th partial row in order, then the 64 sums in order).
__global__ void __launch_bounds__(1024)
    k_rope_dw(const float* __restrict__ part, int blocks, int d, float* __restrict__ dwq, float* __restrict__ dwk,
              int accumulate) {
  __shared__ float sh[64][17];
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4, col = blockIdx.x * 16 + cx;
  float s = 0.f;
  if (col < 2 * d) {
#pragma unroll 8
    for (int r = ry; r < blocks; r += 64) s += part[(int64_t)r * 2 * d + col];
  }
  sh[ry][cx] = s;
  __syncthreads();
  if (ry == 0 && col < 2 * d) {
#pragma unroll
    for (int q = 1; q < 64; ++q) s += sh[q][cx];
    float* o = col < d ? dwq : dwk;
    if (o) {
      const int c = col < d ? col : col - d;
      o[c] = accumulate ? o[c] + s : s;
    }
  }
}

__global__ void __launch_bounds__(kThreads)
    k_rope_table(int64_t n_pos, int32_t rot, double base, double step, float* __restrict__ table) {
  const int half = rot / 2;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (id >= n_pos * half) return;
  const int64_t pos = id / half;
  const int p = (int)(id - pos * half);
  const double angle = (double)pos * (step * pow(base, -2.0 * p / rot));
  table[pos * rot + p] = (float)cos(angle);
  table[pos * rot + half + p] = (float)sin(angle);
}

// ---- host ---------------------------------------------------------------------------
int lanes_of(int d) {
  int g = 2;
  while (8 * g < d) g *= 2;
  return g;
}

// Groups that share a token's heads: a group takes four heads while that leaves
// two waves per SIMD, else fewer.
int slots_of(const hg_rope_desc* D) {
  const int H = D->heads + D->kv_heads, g = lanes_of(D->d);
  for (int per = 4; per > 1; per /= 2) {
    const int s = (int)cdiv(H, per);
    if (D->n * s * g >= (int64_t)64 * 2048) return s;
  }
  return H;
}

int bwd_blocks(const hg_rope_desc* D) {
  const int64_t groups = D->n * slots_of(D), per = kThreads / lanes_of(D->d);
  return (int)std::max<int64_t>(1, std::min<int64_t>(kBwdBlocks, cdiv(groups, per)));
}

int check(const hg_rope_desc* D, const char* what) {
  if (!D) return fail(HG_ERR_ARG, "%s: null descriptor", what);
  if (D->n < 0 || D->heads < 1 || D->kv_heads < 0 || D->d < 1 || D->rot < 0 || D->rot > D->d || D->n_pos < 0)
    return fail(HG_ERR_ARG, "%s: n=%lld heads=%d kv_heads=%d d=%d rot=%d n_pos=%lld", what, (long long)D->n, D->heads,
                D->kv_heads, D->d, D->rot, (long long)D->n_pos);
  if (D->dtype != HG_DTYPE_F32 && D->dtype != HG_DTYPE_BF16) return fail(HG_ERR_ARG, "%s: dtype %d", what, D->dtype);
  if (D->interleaved != 0 && D->interleaved != 1) return fail(HG_ERR_ARG, "%s: interleaved %d", what, D->interleaved);
  if (!(D->eps >= 0.f)) return fail(HG_ERR_ARG, "%s: eps %g", what, (double)D->eps);
  if (D->d % 8 || D->rot % 8 || D->d > kMaxD)
    return fail(HG_ERR_UNSUPPORTED, "%s: d=%d and rot=%d are not multiples of 8 up to %d", what, D->d, D->rot, kMaxD);
  if (D->heads > 1 << 16 || D->kv_heads > 1 << 16 || D->n > ((int64_t)1 << 35) / (D->heads + D->kv_heads))
    return fail(HG_ERR_UNSUPPORTED, "%s: n=%lld tokens of %d heads are too many", what, (long long)D->n,
                D->heads + D->kv_heads);
  return HG_OK;
}

int check_heads(const hg_rope_desc* D, const char* what, const hg_heads* x, int heads, const char* name) {
  if (heads == 0) return HG_OK;
  if (!x || (!x->p && D->n > 0)) return fail(HG_ERR_ARG, "%s: null %s", what, name);
  const int64_t e = D->dtype == HG_DTYPE_F32 ? 4 : 8;
  if ((reinterpret_cast<uintptr_t>(x->p) & 15) || x->token % e || x->head % e)
    return fail(HG_ERR_ARG, "%s: rows of %s are not 16-byte aligned", what, name);
  return HG_OK;
}

Heads heads(const hg_heads* x) { return x ? Heads{x->p, x->token, x->head} : Heads{nullptr, 0, 0}; }

int check_vectors(const hg_rope_desc* D, const char* what, const float* wq, const float* wk, const float* table,
                  const int32_t* pos) {
  if (!pos || (!table && D->rot > 0 && D->n_pos > 0)) return fail(HG_ERR_ARG, "%s: null pointer", what);
  if ((reinterpret_cast<uintptr_t>(wq) | reinterpret_cast<uintptr_t>(wk) | reinterpret_cast<uintptr_t>(table)) & 15)
    return fail(HG_ERR_ARG, "%s: the weights and the table must be 16-byte aligned", what);
  return HG_OK;
}

// A grid has fewer than 2^32 threads.
bool launchable(int64_t groups, int lanes) { return groups <= (((int64_t)1 << 32) - kThreads) / lanes; }

RopeArgs args_of(const hg_rope_desc* D, const hg_heads* q, const hg_heads* k, const float* wq, const float* wk,
                 const float* table, const int32_t* pos) {
  RopeArgs a{};
  a.q = heads(q);
  a.k = heads(D->kv_heads ? k : nullptr);
  a.wq = wq;
  a.wk = wk;
  a.table = table;
  a.pos = pos;
  a.n = D->n;
  a.n_pos = D->n_pos;
  a.hq = D->heads;
  a.hk = D->kv_heads;
  a.d = D->d;
  a.rot = D->rot;
  a.inter = D->interleaved;
  a.slots = slots_of(D);
  a.eps = D->eps;
  return a;
}

template <class T, int G>
int launch(const RopeArgs& a, bool bwd, int blocks, hipStream_t s) {
  if (bwd) {
    HG_LAUNCH("qk_norm_rope_bwd", (k_qk_norm_rope_bwd<T, G, 2>), dim3(blocks), dim3(kThreads), 0, s, a);
  } else {
    HG_LAUNCH("qk_norm_rope", (k_qk_norm_rope<T, G, 4>), dim3((unsigned)cdiv(a.n * a.slots, kThreads / G)),
              dim3(kThreads), 0, s, a);
  }
  return HG_OK;
}

template <class T>
int launch_d(const RopeArgs& a, bool bwd, int blocks, hipStream_t s) {
  switch (lanes_of(a.d)) {
    case 2: return launch<T, 2>(a, bwd, blocks, s);
    case 4: return launch<T, 4>(a, bwd, blocks, s);
    case 8: return launch<T, 8>(a, bwd, blocks, s);
    case 16: return launch<T, 16>(a, bwd, blocks, s);
    default: return launch<T, 32>(a, bwd, blocks, s);
  }
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" int hg_rope_table(int64_t n_pos, int32_t rot, double base, double step, float* table, void* stream) {
  if (n_pos < 0 || rot < 0 || rot % 2 || !(base > 0) || !std::isfinite(base) || !std::isfinite(step))
    return fail(HG_ERR_ARG, "hg_rope_table: n_pos=%lld rot=%d base=%g step=%g", (long long)n_pos, rot, base, step);
  if (rot > kMaxD || n_pos > (int64_t)1 << 31 || (rot > 0 && !launchable(n_pos, rot / 2)))
    return fail(HG_ERR_UNSUPPORTED, "hg_rope_table: n_pos=%lld rot=%d", (long long)n_pos, rot);
  if (n_pos == 0 || rot == 0) return HG_OK;
  if (!table) return fail(HG_ERR_ARG, "hg_rope_table: null pointer");
  HG_LAUNCH("rope_table", k_rope_table, dim3((unsigned)cdiv(n_pos * (rot / 2), kThreads)), dim3(kThreads), 0,
            static_cast<hipStream_t>(stream), n_pos, rot, base, step, table);
  return HG_OK;
}

extern "C" int hg_qk_norm_rope_fwd(const hg_rope_desc* D, const hg_heads* q, const hg_heads* k, const float* wq,
                                   const float* wk, const float* table, const int32_t* pos, const hg_heads* q_out,
                                   const hg_heads* k_out, void* stream) {
  const char* what = "hg_qk_norm_rope_fwd";
  HG_TRY(check(D, what));
  HG_TRY(check_heads(D, what, q, D->heads, "q"));
  HG_TRY(check_heads(D, what, k, D->kv_heads, "k"));
  HG_TRY(check_heads(D, what, q_out, D->heads, "q_out"));
  HG_TRY(check_heads(D, what, k_out, D->kv_heads, "k_out"));
  if (D->n == 0) return HG_OK;
  HG_TRY(check_vectors(D, what, wq, wk, table, pos));
  RopeArgs a = args_of(D, q, k, wq, wk, table, pos);
  if (!launchable(a.n * a.slots, lanes_of(D->d)))
    return fail(HG_ERR_UNSUPPORTED, "%s: n=%lld tokens of %d heads are too many", what, (long long)D->n,
                D->heads + D->kv_heads);
  a.oq = heads(q_out);
  a.ok = heads(D->kv_heads ? k_out : nullptr);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return D->dtype == HG_DTYPE_F32 ? launch_d<float>(a, false, 0, s) : launch_d<bf16_t>(a, false, 0, s);
}

extern "C" size_t hg_qk_norm_rope_bwd_workspace_size(const hg_rope_desc* D) {
  if (check(D, "workspace size") != HG_OK || D->n == 0) return 0;
  Sizer m;
  m.take<float>((int64_t)bwd_blocks(D) * 2 * D->d);
  return m.used;
}

extern "C" int hg_qk_norm_rope_bwd(const hg_rope_desc* D, const hg_heads* q, const hg_heads* k, const float* wq,
                                   const float* wk, const float* table, const int32_t* pos, const hg_heads* dq_out,
                                   const hg_heads* dk_out, const hg_heads* dq, const hg_heads* dk, float* dwq, float* dwk,
                                   int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* what = "hg_qk_norm_rope_bwd";
  HG_TRY(check(D, what));
  if (accumulate != 0 && accumulate != 1) return fail(HG_ERR_ARG, "%s: accumulate %d", what, accumulate);
  const hg_heads* all[6] = {q, k, dq_out, dk_out, dq, dk};
  const char* names[6] = {"q", "k", "dq_out", "dk_out", "dq", "dk"};
  for (int i = 0; i < 6; ++i) HG_TRY(check_heads(D, what, all[i], i & 1 ? D->kv_heads : D->heads, names[i]));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (D->n == 0) {
    if (!accumulate && dwq) HG_TRY(fill_f32(dwq, 0.f, D->d, s));
    if (!accumulate && dwk) HG_TRY(fill_f32(dwk, 0.f, D->d, s));
    return HG_OK;
  }
  HG_TRY(check_vectors(D, what, wq, wk, table, pos));
  RopeArgs a = args_of(D, q, k, wq, wk, table, pos);
  a.gq = heads(dq_out);
  a.gk = heads(D->kv_heads ? dk_out : nullptr);
  a.oq = heads(dq);
  a.ok = heads(D->kv_heads ? dk : nullptr);
  const int blocks = bwd_blocks(D);
  if (dwq || dwk) {
    Sizer need;
    need.take<float>((int64_t)blocks * 2 * D->d);
    if (!ws || ws_bytes < need.used)
      return fail(HG_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need.used);
    if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(HG_ERR_ARG, "%s: the workspace is not 16-byte aligned", what);
    Arena m(ws, ws_bytes);
    a.part = m.take<float>((int64_t)blocks * 2 * D->d);
  }
  HG_TRY(D->dtype == HG_DTYPE_F32 ? launch_d<float>(a, true, blocks, s) : launch_d<bf16_t>(a, true, blocks, s));
  if (a.part)
    HG_LAUNCH("rope_dw", k_rope_dw, dim3((unsigned)cdiv(2 * D->d, 16)), dim3(1024), 0, s, a.part, blocks, D->d, dwq,
              dwk, accumulate);
  return HG_OK;
}
