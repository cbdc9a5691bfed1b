// Group norm with an activation over rows of channels, forward and backward.
//
//   u = (x - mean) rstd,  z = w u + b,  y = act(z)
// with the mean and rstd = 1 / sqrt(var + eps) of a sequence's tokens in a group
// of cg channels; backward, with dz = dy act'(z) and e = w dz:
//   dx = rstd (e - mean(e) - u mean(e u)),  dw = sum dz u,  db = sum dz
//
// A group of a sequence (an item) that some threads can hold is read once: 2^lc
// threads side by side, each with V adjacent channels, times rows of them, each
// with up to R tokens, form the mean, then the squares about it, then the output
// (k_norm_fwd; in the backward the two means, k_norm_bwd).  Items of a wave or
// less reduce by shuffles, larger ones through LDS.  A block's items lie side by
// side, so that whole rows are read.  Larger items are cut into chunks of tokens:
// means and squares of the chunks by the same kernel, joined (k_norm_join), and a
// pass that forms the output (k_norm_apply); in the backward sums of the columns,
// joined, and a pass.
//
// Bound by HBM, the backward with an activation by the vector unit as well (55% of the
// cycles: 16384 rows of 16 x 64 bfloat16 channels 34 us, 3.0 TB/s).  A float32 backward
// of 200003 rows of 128 channels: 51 us for the columns (4.1 TB/s), 48 for the pass
// (6.4); a forward of 512 x 96 tokens of 200 float32 channels 16 us (4.3).
#include <cmath>

#include "hg_gemm.h"
#include "hg_rows4.h"

namespace hg {
namespace {

struct NormArgs {
  Rows x, y;             // y: the output rows (dx in the backward)
  Rows dy;
  const float *w, *b;
  const int32_t* lens;
  float* stats;          // [batch][groups][2]
  float* part;           // chunks' moments, or the blocks' sums of dw and db
  const float* gsum;     // [batch][groups][2] sums of e and of e u (backward pass over chunks)
  int64_t t, ct;         // tokens of a sequence, of a chunk
  int64_t rows;          // sequences times chunks
  int32_t chunks;
  int32_t batch, width, groups, cg;
  int32_t nv;            // cg / V
  int32_t lc, lp;        // log2 of the threads side by side and of an item's threads
  int32_t gper, slabs;   // groups that a block has side by side, blocks of a row
  int32_t rper, row_blocks;  // rows of a block at a time, blocks that share the rows
  int32_t act;
  float eps;
};

template <class T, int V>
__device__ __forceinline__ T* at(const Rows& x, int64_t b, int64_t t, int c) {
  return static_cast<T*>(x.p) + b * x.sb + t * x.st + c;
}

__device__ __forceinline__ int64_t len_of(const NormArgs& a, int64_t b) {
  if (!a.lens) return a.t;
  const int32_t n = a.lens[b];
  return n < 0 ? 0 : (n < a.t ? n : a.t);
}

// act and its slope of V values
template <int ACT, bool G, int V>
__device__ __forceinline__ void act_of(const float (&z)[V], float (&f)[V], float (&d)[V]) {
#pragma unroll
  for (int q = 0; q < V; q += 4) {
    float zz[4], ff[4], dd[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) zz[j] = q + j < V ? z[q + j] : 0.f;
    g_act4<ACT, G>(zz, ff, dd);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (q + j < V) {
        f[q + j] = ff[j];
        if (G) d[q + j] = dd[j];
      }
  }
}

// Sums of N values over the 2^lp threads of an item, in each of them.  More than a
// wave: through sh, which no two calls in a row may share.
template <int N>
__device__ __forceinline__ void item_sum(float (&s)[N], int lp, float (*sh)[N]) {
  const int most = lp < 6 ? lp : 6;
  for (int o = 0; o < most; ++o)
#pragma unroll
    for (int n = 0; n < N; ++n) s[n] += __shfl_xor(s[n], 1 << o, 64);
  if (lp > 6) {
    const int wave = threadIdx.x >> 6, per = 1 << (lp - 6), first = wave & ~(per - 1);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) sh[wave][n] = s[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) s[n] = 0.f;
    for (int q = 0; q < per; ++q)
#pragma unroll
      for (int n = 0; n < N; ++n) s[n] += sh[first + q][n];
  }
}

// The place of a thread in its block's items.
struct Spot {
  int c, r, nr;   // first channel, row lane, row lanes of the item
  int row, g;     // row of the block's rows, group
  bool on;        // the thread has channels
  uint32_t rb;    // block of rows
};
template <int V>
__device__ __forceinline__ Spot spot_of(const NormArgs& a) {
  Spot s;
  const int slot = threadIdx.x >> a.lp, q = threadIdx.x & ((1 << a.lp) - 1), cv = q & ((1 << a.lc) - 1);
  s.r = q >> a.lc;
  s.nr = 1 << (a.lp - a.lc);
  s.rb = blockIdx.x / (uint32_t)a.slabs;
  const int slab = (int)(blockIdx.x - s.rb * (uint32_t)a.slabs);
  s.row = slot / a.gper;
  s.g = slab * a.gper + slot - s.row * a.gper;
  s.on = s.row < a.rper && s.g < a.groups && cv < a.nv;
  s.c = s.g * a.cg + cv * V;
  return s;
}

template <int V>
__device__ __forceinline__ void affine(const NormArgs& a, const Spot& s, float (&w)[V], float (&b)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    w[j] = a.w && s.on ? a.w[s.c + j] : 1.f;
    b[j] = a.b && s.on ? a.b[s.c + j] : 0.f;
  }
}

// CHUNK: only the mean and the sum of squares about it of each chunk of each item.
template <class T, int V, int R, int BT, bool CHUNK>
__global__ void __launch_bounds__(BT) k_norm_fwd(const NormArgs a) {
  __shared__ float sh[2][BT / 64][1];
  const Spot s = spot_of<V>(a);
  float w[V], bias[V];
  if constexpr (!CHUNK) affine<V>(a, s, w, bias);
  for (int64_t i0 = (int64_t)s.rb * a.rper; i0 < a.rows; i0 += (int64_t)a.row_blocks * a.rper) {
    const int64_t i = i0 + s.row;
    const bool in = s.on && i < a.rows;
    const int64_t b = in ? (CHUNK ? i / a.chunks : i) : 0, t0 = CHUNK && in ? (i - b * a.chunks) * a.ct : 0;
    int64_t n = in ? len_of(a, b) - t0 : 0;
    n = n < 0 ? 0 : (CHUNK && n > a.ct ? a.ct : n);
    typename Vec<T, V>::raw x[R];
    float sum[1] = {0.f};
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t t = s.r + k * s.nr;
      if (t < n) x[k] = Vec<T, V>::load(at<T, V>(a.x, b, t0 + t, s.c));
    }
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (s.r + k * s.nr < n)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += Vec<T, V>::get(x[k], j);
    item_sum<1>(sum, a.lp, sh[0]);
    const float inv = n > 0 ? 1.f / (float)(n * a.cg) : 0.f, mean = sum[0] * inv;
    float sq[1] = {0.f};
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (s.r + k * s.nr < n)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = Vec<T, V>::get(x[k], j) - mean;
          sq[0] = fmaf(d, d, sq[0]);
        }
    item_sum<1>(sq, a.lp, sh[1]);
    const bool first = in && (threadIdx.x & ((1 << a.lp) - 1)) == 0;
    if constexpr (CHUNK) {
      if (first) {
        a.part[(i * a.groups + s.g) * 2] = mean;
        a.part[(i * a.groups + s.g) * 2 + 1] = sq[0];
      }
    } else {
      const float rstd = n > 0 ? 1.f / sqrtf(fmaf(sq[0], inv, a.eps)) : 0.f;
      if (first && a.stats) {
        a.stats[(b * a.groups + s.g) * 2] = mean;
        a.stats[(b * a.groups + s.g) * 2 + 1] = rstd;
      }
      if (in)
        g_by_act<true>(a.act, [&](auto act) {
          constexpr int ACT = decltype(act)::value;
#pragma unroll
          for (int k = 0; k < R; ++k) {
            const int64_t t = s.r + k * s.nr;
            if (t >= a.t) break;
            float z[V], f[V], d[V];
#pragma unroll
            for (int j = 0; j < V; ++j) z[j] = fmaf((Vec<T, V>::get(x[k], j) - mean) * rstd, w[j], bias[j]);
            act_of<ACT, false, V>(z, f, d);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = t < n ? f[j] : 0.f;
            Vec<T, V>::put(at<T, V>(a.y, b, t, s.c), f);
          }
        });
    }
  }
}

template <class T, int V, int R, int BT>
__global__ void __launch_bounds__(BT) k_norm_bwd(const NormArgs a) {
  // u stays in registers for the second pass where they last (float32, SiLU: 16384 rows of
  // 16 x 64 channels 43 us, 53 where it is formed again; 512 x 96 tokens of 5 x 40
  // channels, eight of a thread, 55 and 30)
  constexpr bool KEEP = R * V <= 16;
  __shared__ float sh[2][BT / 64][2];
  __shared__ float col[BT * V];
  const Spot s = spot_of<V>(a);
  float w[V], bias[V], dw[V], db[V];
  affine<V>(a, s, w, bias);
#pragma unroll
  for (int j = 0; j < V; ++j) dw[j] = db[j] = 0.f;
  int odd = 0;
  for (int64_t i0 = (int64_t)s.rb * a.rper; i0 < a.rows; i0 += (int64_t)a.row_blocks * a.rper, odd ^= 1) {
    const int64_t b = i0 + s.row;
    const bool in = s.on && b < a.rows;
    const int64_t n = in ? len_of(a, b) : 0;
    typename Vec<T, V>::raw x[R], y[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t t = s.r + k * s.nr;
      if (t < n) {
        x[k] = Vec<T, V>::load(at<T, V>(a.x, b, t, s.c));
        y[k] = Vec<T, V>::load(at<T, V>(a.dy, b, t, s.c));
      }
    }
    const float mean = in ? a.stats[(b * a.groups + s.g) * 2] : 0.f, rstd = in ? a.stats[(b * a.groups + s.g) * 2 + 1] : 0.f;
    float e[R][V], u[KEEP ? R : 1][V], sum[2] = {0.f, 0.f};
    g_by_act<true>(a.act, [&](auto act) {
      constexpr int ACT = decltype(act)::value;
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (s.r + k * s.nr < n) {
          float z[V], f[V], d[V];
#pragma unroll
          for (int j = 0; j < V; ++j) {
            u[KEEP ? k : 0][j] = (Vec<T, V>::get(x[k], j) - mean) * rstd;
            z[j] = fmaf(u[KEEP ? k : 0][j], w[j], bias[j]);
          }
          act_of<ACT, true, V>(z, f, d);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float dz = Vec<T, V>::get(y[k], j) * d[j];
            dw[j] = fmaf(dz, u[KEEP ? k : 0][j], dw[j]);
            db[j] += dz;
            e[k][j] = dz * w[j];
            sum[0] += e[k][j];
            sum[1] = fmaf(e[k][j], u[KEEP ? k : 0][j], sum[1]);
          }
        }
    });
    item_sum<2>(sum, a.lp, sh[odd]);
    const float inv = n > 0 ? 1.f / (float)(n * a.cg) : 0.f, c0 = sum[0] * inv * rstd, c1 = sum[1] * inv * rstd;
    if (in)
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int64_t t = s.r + k * s.nr;
        if (t >= a.t) break;
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float v = KEEP ? u[KEEP ? k : 0][j] : (Vec<T, V>::get(x[k], j) - mean) * rstd;
          o[j] = t < n ? fmaf(rstd, e[k][j], fmaf(-c1, v, -c0)) : 0.f;
        }
        Vec<T, V>::put(at<T, V>(a.y, b, t, s.c), o);
      }
  }
  if (!a.part) return;
  // the block's sums of each channel: over its rows and row lanes, in order
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) col[threadIdx.x * V + j] = h ? db[j] : dw[j];
    __syncthreads();
    const int nc = a.gper * a.cg;
    const int slab = (int)(blockIdx.x - s.rb * (uint32_t)a.slabs), g0 = slab * a.gper;
    for (int c = threadIdx.x; c < nc; c += BT) {
      const int g = c / a.cg, x = c - g * a.cg, cv = x / V, j = x - cv * V;
      if (g0 + g >= a.groups) break;
      float sum = 0.f;
      for (int r = 0; r < a.rper; ++r)
        for (int q = 0; q < s.nr; ++q)
          sum += col[((((r * a.gper + g) << a.lp) + (q << a.lc)) + cv) * V + j];
      a.part[((int64_t)s.rb * 2 + h) * a.width + g0 * a.cg + c] = sum;
    }
  }
}

// Mean and rstd of an item from its chunks' means and squares: a wave each.
__global__ void __launch_bounds__(256) k_norm_join(const NormArgs a, float* __restrict__ stats) {
  const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 6;
  const int lane = threadIdx.x & 63;
  if (id >= (int64_t)a.batch * a.groups) return;
  const int64_t b = id / a.groups;
  const int g = (int)(id - b * a.groups);
  const int64_t n = len_of(a, b);
  auto sum = [](double v) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o, 64);
    return v;
  };
  const float* p = a.part + (b * a.chunks * a.groups + g) * 2;
  const int chunks = (int)((n + a.ct - 1) / a.ct);
  double m = 0;
  for (int k = lane; k < chunks; k += 64) {
    const int64_t k0 = k * a.ct, in = n - k0 < a.ct ? n - k0 : a.ct;
    m += (double)p[(int64_t)k * a.groups * 2] * (double)in;
  }
  const double mean = n > 0 ? sum(m) / (double)n : 0;
  double q = 0;
  for (int k = lane; k < chunks; k += 64) {
    const int64_t k0 = k * a.ct, in = n - k0 < a.ct ? n - k0 : a.ct;
    const double d = (double)p[(int64_t)k * a.groups * 2] - mean;
    q += (double)p[(int64_t)k * a.groups * 2 + 1] + d * d * (double)(in * a.cg);
  }
  q = sum(q);
  if (lane == 0) {
    stats[id * 2] = (float)mean;
    stats[id * 2 + 1] = n > 0 ? (float)(1.0 / sqrt(q / (double)(n * a.cg) + (double)a.eps)) : 0.f;
  }
}

constexpr int kApply = 8;  // tokens of a thread

// The output from the statistics: y, or with BACK dx.
template <class T, int V, bool BACK>
__global__ void __launch_bounds__(256) k_norm_apply(const NormArgs a, const float* __restrict__ stats) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int cols = a.width / V;
  const int64_t tile = id / cols, per = (a.t + kApply - 1) / kApply, b = tile / per;
  const int c = (int)(id - tile * cols) * V;
  if (b >= a.batch) return;
  const int64_t t0 = (tile - b * per) * kApply, n = len_of(a, b);
  const int g = c / a.cg;
  const float mean = stats[(b * a.groups + g) * 2], rstd = stats[(b * a.groups + g) * 2 + 1];
  float c0 = 0.f, c1 = 0.f;
  if (BACK) {
    const float inv = n > 0 ? (float)(1.0 / (double)(n * a.cg)) : 0.f;
    c0 = a.gsum[(b * a.groups + g) * 2] * inv * rstd;
    c1 = a.gsum[(b * a.groups + g) * 2 + 1] * inv * rstd;
  }
  float w[V], bias[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    w[j] = a.w ? a.w[c + j] : 1.f;
    bias[j] = a.b ? a.b[c + j] : 0.f;
  }
  typename Vec<T, V>::raw x[kApply], dy[kApply];
#pragma unroll
  for (int k = 0; k < kApply; ++k)
    if (t0 + k < n) {
      x[k] = Vec<T, V>::load(at<T, V>(a.x, b, t0 + k, c));
      if constexpr (BACK) dy[k] = Vec<T, V>::load(at<T, V>(a.dy, b, t0 + k, c));
    }
  g_by_act<true>(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
#pragma unroll
    for (int k = 0; k < kApply; ++k) {
      if (t0 + k >= a.t) break;
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = 0.f;
      if (t0 + k < n) {
        float u[V], z[V], f[V], d[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          u[j] = (Vec<T, V>::get(x[k], j) - mean) * rstd;
          z[j] = fmaf(u[j], w[j], bias[j]);
        }
        act_of<ACT, BACK, V>(z, f, d);
#pragma unroll
        for (int j = 0; j < V; ++j)
          o[j] = BACK ? fmaf(rstd, Vec<T, V>::get(dy[k], j) * d[j] * w[j], fmaf(-c1, u[j], -c0)) : f[j];
      }
      Vec<T, V>::put(at<T, V>(a.y, b, t0 + k, c), o);
    }
  });
}

// Sums of dz u and of dz of each column over a chunk of a sequence's tokens:
// 2^lc threads side by side, 256 >> lc rows of them, four tokens in flight.
template <class T, int V>
__global__ void __launch_bounds__(256) k_norm_cols(const NormArgs a) {
  __shared__ float sh[256 * V];
  const int cv = threadIdx.x & ((1 << a.lc) - 1), r = threadIdx.x >> a.lc, nr = 256 >> a.lc;
  const uint32_t i = blockIdx.x / (uint32_t)a.slabs;
  const int slab = (int)(blockIdx.x - i * (uint32_t)a.slabs);
  const int64_t b = i / (uint32_t)a.chunks, t0 = (i - b * a.chunks) * a.ct;
  const int c = ((slab << a.lc) + cv) * V;
  const bool on = c < a.width;
  int64_t n = len_of(a, b) - t0;
  n = n < a.ct ? n : a.ct;
  const int g = on ? c / a.cg : 0;
  const float mean = a.stats[(b * a.groups + g) * 2], rstd = a.stats[(b * a.groups + g) * 2 + 1];
  float w[V], bias[V], dw[V], db[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    w[j] = a.w && on ? a.w[c + j] : 1.f;
    bias[j] = a.b && on ? a.b[c + j] : 0.f;
    dw[j] = db[j] = 0.f;
  }
  g_by_act<true>(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    for (int64_t t = r; on && t < n; t += 4 * nr) {
      typename Vec<T, V>::raw x[4], dy[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (t + k * nr < n) {
          x[k] = Vec<T, V>::load(at<T, V>(a.x, b, t0 + t + k * nr, c));
          dy[k] = Vec<T, V>::load(at<T, V>(a.dy, b, t0 + t + k * nr, c));
        }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (t + k * nr < n) {
          float u[V], z[V], f[V], d[V];
#pragma unroll
          for (int j = 0; j < V; ++j) {
            u[j] = (Vec<T, V>::get(x[k], j) - mean) * rstd;
            z[j] = fmaf(u[j], w[j], bias[j]);
          }
          act_of<ACT, true, V>(z, f, d);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float dz = Vec<T, V>::get(dy[k], j) * d[j];
            dw[j] = fmaf(dz, u[j], dw[j]);
            db[j] += dz;
          }
        }
    }
  });
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) sh[threadIdx.x * V + j] = h ? db[j] : dw[j];
    __syncthreads();
    for (int q = threadIdx.x; q < V << a.lc; q += 256) {
      const int col = (slab << a.lc) * V + q;
      if (col >= a.width) break;
      float sum = 0.f;
      for (int k = 0; k < nr; ++k) sum += sh[((k << a.lc) * V) + q];
      a.part[((int64_t)i * 2 + h) * a.width + col] = sum;
    }
  }
}

// out[b][h][c] = sum over rows of part[b][row][h][c]: 16 columns a block, 64 threads
// a column (every 64th row in order, then the 64 sums in order).
__global__ void __launch_bounds__(1024)
    k_norm_fold(const float* __restrict__ part, int64_t rows, int32_t cols, float* __restrict__ out) {
  __shared__ float sh[64][17];
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const uint32_t per = ((uint32_t)cols + 15) / 16;
  const int64_t b = blockIdx.x / per;
  const int c = (int)(blockIdx.x - b * per) * 16 + cx;
  part += b * rows * cols;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t r = ry; r < rows; r += 64) s += part[r * cols + c];
  }
  sh[ry][cx] = s;
  __syncthreads();
  if (ry == 0 && c < cols) {
#pragma unroll
    for (int q = 1; q < 64; ++q) s += sh[q][cx];
    out[b * cols + c] = s;
  }
}

// dw and db over rows of part [rows][2][width], and with gsum the sums of e u and
// of e of each item from one row of part for each sequence.  The first
// ceil(2 width / 16) blocks do the former, a wave of the others an item each.
__global__ void __launch_bounds__(1024)
    k_norm_grads(const float* __restrict__ part, int64_t rows, int32_t width, int32_t groups, const float* __restrict__ w,
                 float* __restrict__ dw, float* __restrict__ db, int32_t accumulate, float* __restrict__ gsum) {
  __shared__ float sh[64][17];
  const uint32_t cols = 2 * (uint32_t)width, first = (cols + 15) / 16;
  if (blockIdx.x >= first) {
    const int64_t id = (int64_t)(blockIdx.x - first) * 16 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, cg = width / groups;
    if (id >= rows * groups) return;
    const int64_t b = id / groups;
    const int g = (int)(id - b * groups);
    const float* p = part + b * cols + g * cg;
    float s0 = 0.f, s1 = 0.f;
    for (int c = lane; c < cg; c += 64) {
      const float x = w ? w[g * cg + c] : 1.f;
      s1 = fmaf(x, p[c], s1);
      s0 = fmaf(x, p[width + c], s0);
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) s0 += __shfl_xor(s0, o, 64), s1 += __shfl_xor(s1, o, 64);
    if (lane == 0) gsum[id * 2] = s0, gsum[id * 2 + 1] = s1;
    return;
  }
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const uint32_t c = blockIdx.x * 16 + cx;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t r = ry; r < rows; r += 64) s += part[r * cols + c];
  }
  sh[ry][cx] = s;
  __syncthreads();
  if (ry == 0 && c < cols) {
#pragma unroll
    for (int q = 1; q < 64; ++q) s += sh[q][cx];
    float* o = c < (uint32_t)width ? dw : db;
    if (o) {
      const uint32_t k = c < (uint32_t)width ? c : c - width;
      o[k] = accumulate ? o[k] + s : s;
    }
  }
}

// ---- host ---------------------------------------------------------------------------
int log2_up(int64_t n) {
  int l = 0;
  while (((int64_t)1 << l) < n) ++l;
  return l;
}

// How a call is laid out.
struct Plan {
  int v;          // channels of a thread
  int r;          // tokens of a thread (1, 2, 4, 8)
  int bt;         // threads of a block
  bool chunked;
  NormArgs a;     // sizes only
  int64_t blocks;
};

// Widest vector that the groups are made of.
int vec_of(const hg_group_norm_desc* A) {
  const int cg = A->width / A->groups;
  if (A->dtype == HG_DTYPE_BF16) return cg % 8 == 0 ? 8 : cg % 4 == 0 ? 4 : 1;
  return cg % 4 == 0 ? 4 : 1;
}

constexpr int kMostRows = 8;

// Items on 2^lp threads each, `bt` threads a block, rows shared by at most `most` blocks.
void lay_out(Plan& p, int64_t rows, int64_t most) {
  NormArgs& a = p.a;
  const int slots = p.bt >> a.lp;
  a.gper = std::min(a.groups, slots);
  a.slabs = (int32_t)cdiv(a.groups, a.gper);
  a.rper = slots / a.gper;
  a.rows = rows;
  a.row_blocks = (int32_t)std::max<int64_t>(1, std::min(cdiv(rows, a.rper), most / a.slabs));
  p.blocks = (int64_t)a.row_blocks * a.slabs;
}

Plan plan_of(const hg_group_norm_desc* A, bool bwd) {
  Plan p{};
  NormArgs& a = p.a;
  a.t = a.ct = A->t;
  a.chunks = 1;
  a.batch = A->batch;
  a.width = A->width;
  a.groups = A->groups;
  a.cg = A->width / A->groups;
  a.act = A->act;
  a.eps = A->eps;
  p.v = vec_of(A);
  a.nv = a.cg / p.v;
  a.lc = log2_up(a.nv);
  // An item's threads: up to 256 of four or eight tokens each, else up to 1024 of eight
  // (in the backward, which holds three times as much, of one or two); else chunks.  Few
  // such items too: one of 1000 float32 tokens of 16 channels takes 12 us, 18 in chunks.
  const int64_t t = std::max<int64_t>(A->t, 1);
  const int lr4 = log2_up(cdiv(t, 4)), lr8 = log2_up(cdiv(t, kMostRows)), lrb = log2_up(cdiv(t, p.v == 8 ? 1 : 2));
  const int lr = a.lc + lr4 <= 8 ? lr4 : a.lc + lr8 <= 8 || !bwd ? lr8 : lrb;
  p.chunked = a.lc + lr > 10;
  if (!p.chunked) {
    a.lp = a.lc + lr;
    p.r = 1 << std::min(3, log2_up(cdiv(t, (int64_t)1 << lr)));
    p.bt = a.lp <= 8 ? 256 : 1024;
    // A block fetches w and b once, and each block of the backward has a row of partial sums
    // of dw and db: few blocks, but enough to fill the chip.  Forward, 16384 rows of 16 x 64
    // channels: bfloat16 30 us with 2048, 28 with 1024, 37 with 4096, 62 with one for every two
    // rows, float32 29, 33, 29 and 37; of 1024 threads, 4096 bfloat16 rows of 4096 channels 34 us
    // with 512, 42 with 1024, 63 with one for each.  Backward, the same rows: bfloat16 37 us with
    // 1024, 36 with 512, 44 with 2048, float32 44, 57 and 52; of 1024 threads, 4096 rows of 8192
    // bfloat16 channels 74 us with 256, 90 with 512, 118 with 128.  Single channels a thread are
    // few bytes in flight and take more: 30000 bfloat16 rows of 32 x 25 channels forward 124 us
    // with 4096, 133 with 2048, 161 with one for each; backward, 20000 such rows 71 us with 2048,
    // 90 with 1024, 69 with 4096, 100000 float32 ones of 5 x 25 87, 125 and 93.
    if (bwd) {
      lay_out(p, A->batch, p.bt > 256 ? 256 : p.v == 1 ? 2048 : 1024);
    } else {
      lay_out(p, A->batch, p.bt > 256 ? 512 : p.v == 1 ? 4096 : 2048);
    }
    return p;
  }
  p.r = kMostRows;
  p.bt = 256;
  if (bwd) {
    // columns: a slab of 2^lc threads, chunks so that the blocks fill the chip (200003 rows of
    // 128 float32 channels 110 us with 1024 blocks, 108 with 512, 111 with 2048; 64 x 5000 of
    // 128 bfloat16 channels 97, 96 and 93)
    const int64_t cols = A->width / p.v;
    a.lc = std::min(6, log2_up(cols));
    a.slabs = (int32_t)cdiv(cols, (int64_t)1 << a.lc);
    const int64_t rl = 256 >> a.lc, want = std::max<int64_t>(1, 1024 / std::max<int64_t>(1, (int64_t)A->batch * a.slabs));
    a.ct = std::max(cdiv(t, want), 4 * rl);
    a.chunks = (int32_t)cdiv(t, a.ct);
    a.rows = (int64_t)A->batch * a.chunks;
    p.blocks = a.rows * a.slabs;
    return p;
  }
  a.lp = std::max(8, std::min(a.lc, 10));
  if (a.lp > 8) p.bt = 1024;
  a.ct = ((int64_t)1 << (a.lp - a.lc)) * kMostRows;
  a.chunks = (int32_t)cdiv(t, a.ct);
  lay_out(p, (int64_t)A->batch * a.chunks, (int64_t)1 << 21);
  return p;
}

struct Bufs {
  float *part = nullptr, *stats = nullptr, *cols = nullptr, *gsum = nullptr;
};
template <class Mem>
Bufs take(const Plan& p, bool bwd, Mem& m) {
  const NormArgs& a = p.a;
  Bufs b;
  if (!bwd) {
    b.part = m.template take<float>(p.chunked ? a.rows * a.groups * 2 : 0);
    b.stats = m.template take<float>(p.chunked ? (int64_t)a.batch * a.groups * 2 : 0);
    return b;
  }
  b.part = m.template take<float>((p.chunked ? a.rows : (int64_t)a.row_blocks) * 2 * a.width);
  b.cols = m.template take<float>(p.chunked && a.chunks > 1 ? (int64_t)a.batch * 2 * a.width : 0);
  b.gsum = m.template take<float>(p.chunked ? (int64_t)a.batch * a.groups * 2 : 0);
  return b;
}

int check(const hg_group_norm_desc* A, const char* what) {
  if (!A) return fail(HG_ERR_ARG, "%s: null descriptor", what);
  if (A->t < 0 || A->batch < 0 || A->width < 1 || A->groups < 1 || A->width % A->groups)
    return fail(HG_ERR_ARG, "%s: batch=%d t=%lld width=%d groups=%d", what, A->batch, (long long)A->t, A->width, A->groups);
  if (A->dtype != HG_DTYPE_F32 && A->dtype != HG_DTYPE_BF16) return fail(HG_ERR_ARG, "%s: dtype %d", what, A->dtype);
  if (A->act < HG_ACT_NONE || A->act > HG_ACT_GELU) return fail(HG_ERR_ARG, "%s: act %d", what, A->act);
  if (!(A->eps > 0.f) || !std::isfinite(A->eps)) return fail(HG_ERR_ARG, "%s: eps %g", what, (double)A->eps);
  // channels of a thread that are one by one reach 1024 side by side
  const int64_t nv = A->width / A->groups / vec_of(A);
  if (nv > 1024) return fail(HG_ERR_UNSUPPORTED, "%s: groups of %d channels", what, A->width / A->groups);
  // (a grid has fewer than 2^32 threads)
  if (A->t > (int64_t)1 << 40 || A->width > 1 << 20 ||
      (A->t > 0 && (int64_t)A->batch * A->width / vec_of(A) >= ((int64_t)1 << 34) / A->t) || (int64_t)A->batch * A->width >= (int64_t)1 << 32)
    return fail(HG_ERR_UNSUPPORTED, "%s: %d sequences of %lld tokens and %d channels are too many", what, A->batch,
                (long long)A->t, A->width);
  return HG_OK;
}

int check_grid(const Plan& p, const hg_group_norm_desc* A, const char* what) {
  if (p.blocks * p.bt >= (int64_t)1 << 32)
    return fail(HG_ERR_UNSUPPORTED, "%s: %d sequences of %lld tokens and %d channels are too many", what, A->batch,
                (long long)A->t, A->width);
  return HG_OK;
}

unsigned apply_blocks(const NormArgs& a, int v) {
  return (unsigned)cdiv((int64_t)a.batch * cdiv(a.t, kApply) * (a.width / v), 256);
}

template <class T, int V>
int launch_fwd(const Plan& p, const NormArgs& a, const Bufs& b, hipStream_t s) {
  const dim3 grid((unsigned)p.blocks);
  if (!p.chunked) {
    const auto by_r = [&](auto bt) {
      constexpr int BT = decltype(bt)::value;
      const char* name = "group_norm";
      switch (p.r) {
        case 1: HG_LAUNCH(name, (k_norm_fwd<T, V, 1, BT, false>), grid, dim3(BT), 0, s, a); break;
        case 2: HG_LAUNCH(name, (k_norm_fwd<T, V, 2, BT, false>), grid, dim3(BT), 0, s, a); break;
        case 4: HG_LAUNCH(name, (k_norm_fwd<T, V, 4, BT, false>), grid, dim3(BT), 0, s, a); break;
        default: HG_LAUNCH(name, (k_norm_fwd<T, V, 8, BT, false>), grid, dim3(BT), 0, s, a);
      }
      return HG_OK;
    };
    return p.bt == 256 ? by_r(std::integral_constant<int, 256>{}) : by_r(std::integral_constant<int, 1024>{});
  }
  if (p.bt == 256) {
    HG_LAUNCH("group_norm_chunks", (k_norm_fwd<T, V, kMostRows, 256, true>), grid, dim3(256), 0, s, a);
  } else {
    HG_LAUNCH("group_norm_chunks", (k_norm_fwd<T, V, kMostRows, 1024, true>), grid, dim3(1024), 0, s, a);
  }
  float* stats = a.stats ? a.stats : b.stats;
  HG_LAUNCH("group_norm_join", k_norm_join, dim3((unsigned)cdiv((int64_t)a.batch * a.groups, 4)), dim3(256), 0, s, a, stats);
  HG_LAUNCH("group_norm_apply", (k_norm_apply<T, V, false>), dim3(apply_blocks(a, V)), dim3(256), 0, s, a, stats);
  return HG_OK;
}

template <class T, int V>
int launch_bwd(const Plan& p, NormArgs a, const Bufs& b, float* dw, float* db, int accumulate, hipStream_t s) {
  const dim3 grid((unsigned)p.blocks);
  const unsigned first = (unsigned)cdiv(2 * (int64_t)a.width, 16);
  if (!p.chunked) {
    if (!dw && !db) a.part = nullptr;
    const char* name = "group_norm_bwd";
    if (p.bt == 256) {
      switch (p.r) {
        case 1: HG_LAUNCH(name, (k_norm_bwd<T, V, 1, 256>), grid, dim3(256), 0, s, a); break;
        case 2: HG_LAUNCH(name, (k_norm_bwd<T, V, 2, 256>), grid, dim3(256), 0, s, a); break;
        case 4: HG_LAUNCH(name, (k_norm_bwd<T, V, 4, 256>), grid, dim3(256), 0, s, a); break;
        default: HG_LAUNCH(name, (k_norm_bwd<T, V, 8, 256>), grid, dim3(256), 0, s, a);
      }
    } else if (p.r == 1) {
      HG_LAUNCH(name, (k_norm_bwd<T, V, 1, 1024>), grid, dim3(1024), 0, s, a);
    } else {
      HG_LAUNCH(name, (k_norm_bwd<T, V < 8 ? V : 4, 2, 1024>), grid, dim3(1024), 0, s, a);  // (never with eight channels)
    }
    if (dw || db)
      HG_LAUNCH("group_norm_grads", k_norm_grads, dim3(first), dim3(1024), 0, s, b.part, (int64_t)a.row_blocks, a.width,
                a.groups, a.w, dw, db, accumulate, nullptr);
    return HG_OK;
  }
  HG_LAUNCH("group_norm_cols", (k_norm_cols<T, V>), grid, dim3(256), 0, s, a);
  const float* cols = b.part;
  if (a.chunks > 1) {
    HG_LAUNCH("group_norm_fold", k_norm_fold, dim3((unsigned)(a.batch * (int64_t)first)), dim3(1024), 0, s, b.part,
              (int64_t)a.chunks, 2 * a.width, b.cols);
    cols = b.cols;
  }
  HG_LAUNCH("group_norm_grads", k_norm_grads, dim3(first + (unsigned)cdiv((int64_t)a.batch * a.groups, 16)), dim3(1024), 0, s,
            cols, (int64_t)a.batch, a.width, a.groups, a.w, dw, db, accumulate, b.gsum);
  a.gsum = b.gsum;
  HG_LAUNCH("group_norm_bwd_apply", (k_norm_apply<T, V, true>), dim3(apply_blocks(a, V)), dim3(256), 0, s, a, a.stats);
  return HG_OK;
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" size_t hg_group_norm_fwd_workspace_size(const hg_group_norm_desc* A) {
  if (check(A, "workspace size") != HG_OK || A->batch == 0 || A->t == 0) return 0;
  Sizer m;
  take(plan_of(A, false), false, m);
  return m.used;
}

extern "C" size_t hg_group_norm_bwd_workspace_size(const hg_group_norm_desc* A) {
  if (check(A, "workspace size") != HG_OK || A->batch == 0 || A->t == 0) return 0;
  Sizer m;
  take(plan_of(A, true), true, m);
  return m.used;
}

extern "C" int hg_group_norm_fwd(const hg_group_norm_desc* A, const hg_heads* x, const float* w, const float* b,
                                 const int32_t* lens, const hg_heads* y, float* stats, void* ws, size_t ws_bytes,
                                 void* stream) {
  const char* what = "hg_group_norm_fwd";
  HG_TRY(check(A, what));
  HG_TRY(check_rows(what, x, "x", false, A->batch, A->t, A->width, A->dtype));
  HG_TRY(check_rows(what, y, "y", true, A->batch, A->t, A->width, A->dtype));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (A->batch == 0) return HG_OK;
  if (A->t == 0) return stats ? fill_f32(stats, 0.f, (int64_t)A->batch * A->groups * 2, s) : HG_OK;
  if (rows_meet(y, x, A->batch, A->t, A->width, A->dtype)) return fail(HG_ERR_ARG, "%s: y overlaps x", what);
  const Plan p = plan_of(A, false);
  HG_TRY(check_grid(p, A, what));
  Sizer need;
  take(p, false, need);
  HG_TRY(check_workspace(what, ws, ws_bytes, need.used));
  Arena m(ws, ws_bytes);
  const Bufs bufs = take(p, false, m);
  NormArgs a = p.a;
  a.x = rows_of(x);
  a.y = rows_of(y);
  a.w = w;
  a.b = b;
  a.lens = lens;
  a.stats = stats;
  a.part = bufs.part;
  if (A->dtype == HG_DTYPE_F32) return p.v == 4 ? launch_fwd<float, 4>(p, a, bufs, s) : launch_fwd<float, 1>(p, a, bufs, s);
  return p.v == 8   ? launch_fwd<bf16_t, 8>(p, a, bufs, s)
         : p.v == 4 ? launch_fwd<bf16_t, 4>(p, a, bufs, s)
                    : launch_fwd<bf16_t, 1>(p, a, bufs, s);
}

extern "C" int hg_group_norm_bwd(const hg_group_norm_desc* A, const hg_heads* x, const float* w, const float* b,
                                 const int32_t* lens, const float* stats, const hg_heads* dy, const hg_heads* dx, float* dw,
                                 float* db, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const char* what = "hg_group_norm_bwd";
  HG_TRY(check(A, what));
  if (accumulate != 0 && accumulate != 1) return fail(HG_ERR_ARG, "%s: accumulate %d", what, accumulate);
  HG_TRY(check_rows(what, x, "x", false, A->batch, A->t, A->width, A->dtype));
  HG_TRY(check_rows(what, dy, "dy", false, A->batch, A->t, A->width, A->dtype));
  HG_TRY(check_rows(what, dx, "dx", true, A->batch, A->t, A->width, A->dtype));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (A->batch == 0 || A->t == 0) {
    if (!accumulate && dw) HG_TRY(fill_f32(dw, 0.f, A->width, s));
    if (!accumulate && db) HG_TRY(fill_f32(db, 0.f, A->width, s));
    return HG_OK;
  }
  if (!stats) return fail(HG_ERR_ARG, "%s: null stats", what);
  for (const hg_heads* v : {x, dy})
    if (rows_meet(dx, v, A->batch, A->t, A->width, A->dtype)) return fail(HG_ERR_ARG, "%s: dx overlaps an input", what);
  const size_t vec = (size_t)A->width * 4;
  if (ranges_meet(dw, vec, w, vec) || ranges_meet(dw, vec, b, vec) || ranges_meet(dw, vec, db, vec) || ranges_meet(db, vec, w, vec) ||
      ranges_meet(db, vec, b, vec))
    return fail(HG_ERR_ARG, "%s: a gradient's buffer is another of the call's", what);
  const Plan p = plan_of(A, true);
  HG_TRY(check_grid(p, A, what));
  Sizer need;
  take(p, true, need);
  HG_TRY(check_workspace(what, ws, ws_bytes, need.used));
  Arena m(ws, ws_bytes);
  const Bufs bufs = take(p, true, m);
  NormArgs a = p.a;
  a.x = rows_of(x);
  a.dy = rows_of(dy);
  a.y = rows_of(dx);
  a.w = w;
  a.b = b;
  a.lens = lens;
  a.stats = const_cast<float*>(stats);
  a.part = bufs.part;
  if (A->dtype == HG_DTYPE_F32)
    return p.v == 4 ? launch_bwd<float, 4>(p, a, bufs, dw, db, accumulate, s) : launch_bwd<float, 1>(p, a, bufs, dw, db, accumulate, s);
  return p.v == 8   ? launch_bwd<bf16_t, 8>(p, a, bufs, dw, db, accumulate, s)
         : p.v == 4 ? launch_bwd<bf16_t, 4>(p, a, bufs, dw, db, accumulate, s)
                    : launch_bwd<bf16_t, 1>(p, a, bufs, dw, db, accumulate, s);
}
