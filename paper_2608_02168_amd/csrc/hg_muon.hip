// One update of matrices along their orthogonalised momentum.
//
//   M = mu M + G,  U = G + mu M or M,  X = U / max(|U|, eps)
//   `steps` times:  A = X X^T,  B = q A + s A A,  X = p X + B X
//   W = (1 - lr wd) W - lr scale X
// (tall matrices: A = X^T X, X = p X + X B), (p, q, s) = (3.4445, -4.7750, 2.0315):
// singular values go through x (p + q x^2 + s x^4), which keeps [0, 1.21] in
// [0, 1.21] and takes small ones up by p a step.
//
// X, A and B are held in two fp16 parts, the high part and what its rounding left (a
// product is then hi hi + hi lo + lo hi, as in the row transforms).  Since no entry
// of X exceeds 1.21, of A 1.47 and of B 2.81, fixed powers of two take them to the
// top of fp16's range, exactly.  Sums are float32.  bfloat16 matrices too: with the
// high part alone, off by 2^-12 of an entry, a step's noise in directions that a
// gradient leaves empty grows by p with each step after it, to 0.03 of X's norm
// where min / 8 directions hold it and 0.1 for rank one (a third of the products:
// 4096 x 8192 in 2.5 ms, 6.2 so).
//
// Each product runs on the fp16 MFMA in tiles, with the tile loads of the linear
// map's products (hg_gemm.h): X is read as it lies, by rows or with k as the row
// index.  A and A A are symmetric: only tiles on and below the diagonal are
// formed, and written twice.  The sums q A + s A A and p X + B X and the update of
// W are the products' epilogues, so a step is three launches (and where the last tiles'
// k is cut, the sums of the parts).  Bound by the MFMA: a step of 4096 x 8192 is 362 us
// for A, 186 for B and 670 for B X (1.1, 1.1 and 1.2 PFLOP/s of fp16 products; a large
// library product 1.2), of 1024 x 5632 34, 16 and 50 (0.5, 0.2 and 0.7 PFLOP/s; the
// tiles are few, and 9 and 6 of it add parts of k).
//
// The iteration with these three coefficients and five steps is a published method (K.
// Jordan and others, 2024: an optimizer for hidden layers).
#include <cmath>

#include "hg_gemm.h"
#include "hg_rows4.h"

namespace hg {
namespace {

constexpr float kP = 3.4445f, kQ = -4.7750f, kS = 2.0315f;
// powers of two of the stored values
constexpr int kXe = 14, kAe = 15, kBe = 14;
constexpr float pow2(int e) { return e >= 0 ? (float)(1ll << e) : 1.f / (float)(1ll << -e); }

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// One stored matrix of rows x cols values, `step` 16-bit values from one matrix of
// the call to the next.  A row holds its columns up to a multiple of 32, zeros from
// cols on; each 32 high parts are followed by their low parts, so that a tile's
// 128-byte rows are 32 columns in two parts.
struct Stored {
  uint16_t* p;
  int64_t step;
  int32_t rows, cols;
  int32_t pad;  // columns with their padding
  int32_t ld;   // values of a row
};
__device__ __forceinline__ int64_t spot(const Stored& o, int r, int c) {
  return (int64_t)r * o.ld + (c >> 5) * 64 + (c & 31);
}

struct MuonArgs {
  Stored a, b;          // operands
  Stored c;             // what the epilogue adds: A for B, X for the next X
  Stored o;             // what it writes
  void* W;              // or the update of W [count][M][N]
  int32_t M, N, K;      // of the product
  int32_t tiles_m, tiles_n, tiles;  // tiles of one matrix
  uint32_t full;        // tiles of the call that one block takes; of the others, each `pieces` blocks a part of k
  int32_t pieces;
  float* part;          // [blocks of parts][BM BN] their sums
  float zs, cs;         // out = zs z + cs c
  float ws, us;         // W = ws W - us (zs z + cs c)
};

enum { kEpiSym = 0, kEpiSymAdd = 1, kEpiAdd = 2, kEpiUpdate = 3 };

// The parts of four adjacent values (of the first of them) of a row.
__device__ __forceinline__ void put4(uint16_t* p, const float (&v)[4]) {
  f16x4 h, l;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h[q] = (_Float16)v[q];
    l[q] = (_Float16)(v[q] - (float)h[q]);
  }
  *reinterpret_cast<f16x4*>(p) = h;
  *reinterpret_cast<f16x4*>(p + 32) = l;
}
__device__ __forceinline__ void put1(uint16_t* p, float v) {
  const _Float16 h = (_Float16)v;
  *p = __builtin_bit_cast(uint16_t, h);
  p[32] = __builtin_bit_cast(uint16_t, (_Float16)(v - (float)h));
}
// Tile (row, column) of tile id of the lower triangle of tm tile rows, in the order
// of g_tile_of: each XCD takes one contiguous share of a walk that goes down eight
// tile rows before it moves to the next tile column.
__device__ __forceinline__ uint32_t row_of_tri(uint32_t id) {
  uint32_t i = (uint32_t)((sqrtf(8.f * (float)id + 1.f) - 1.f) * 0.5f);
  while ((i + 1) * (i + 2) / 2 <= id) ++i;
  while (i * (i + 1) / 2 > id) --i;
  return i;
}
__device__ __forceinline__ void tri_of(uint32_t id, uint32_t tm, uint32_t& im, uint32_t& in) {
  const uint32_t n = tm * (tm + 1) / 2, per = n / 8, more = n % 8, x = id % 8;
  const uint32_t i = x * per + (x < more ? x : more) + id / 8;
  // rows 8 b .. of a band: 8 b whole columns, then a triangle; the bands before have 32 b^2 + 4 b tiles
  uint32_t b = (uint32_t)((sqrtf(16.f + 128.f * (float)i) - 4.f) / 64.f);
  while (32 * (b + 1) * (b + 1) + 4 * (b + 1) <= i) ++b;
  while (32 * b * b + 4 * b > i) --b;
  const uint32_t r = i - (32 * b * b + 4 * b), rows = tm - 8 * b < 8 ? tm - 8 * b : 8;
  if (r < rows * 8 * b) {
    im = 8 * b + r % rows;
    in = r / rows;
  } else {
    const uint32_t t = r - rows * 8 * b, y = row_of_tri(t);
    im = 8 * b + y;
    in = 8 * b + t - y * (y + 1) / 2;
  }
}

// A tile of the call: its matrix, row and column.
template <int EPI>
__device__ __forceinline__ void tile_of(const MuonArgs& p, uint32_t tile, uint32_t& mat, uint32_t& im, uint32_t& in) {
  mat = tile / (uint32_t)p.tiles;
  const uint32_t id = tile - mat * (uint32_t)p.tiles;
  if constexpr (EPI <= kEpiSymAdd) {
    tri_of(id, p.tiles_m, im, in);
  } else {
    g_tile_of(id, p.tiles_m, p.tiles_n, 8, im, in);
  }
}

// What the epilogue of columns n .. n + 3 of row m reads: of X or A, and of W.  All
// of a row of blocks is loaded before the first is written: the compiler keeps loads
// behind stores that may be to the same place, and would wait for each.
template <int EPI, class T>
struct Beside {
  f16x4 h, l;
  typename Vec<T, 4>::raw w;
  __device__ __forceinline__ void load(const MuonArgs& p, uint32_t mat, int m, int n) {
    if constexpr (EPI != kEpiSym) {
      if (m < p.M && n < p.c.pad) {
        const uint16_t* x = p.c.p + mat * p.c.step + spot(p.c, m, n);
        h = *reinterpret_cast<const f16x4*>(x);
        l = *reinterpret_cast<const f16x4*>(x + 32);
      }
    }
    if constexpr (EPI == kEpiUpdate)
      if (m < p.M && n + 4 <= p.N) w = Vec<T, 4>::load(static_cast<const T*>(p.W) + ((int64_t)mat * p.M + m) * p.N + n);
  }
};

// The epilogue of columns n .. n + 3 of row m; mirror: below the diagonal of a
// symmetric result, whose transpose is written too.
template <int EPI, class T>
__device__ __forceinline__ void finish(const MuonArgs& p, uint32_t mat, int m, int n, bool mirror, const f32x4& z,
                                       const Beside<EPI, T>& x) {
  constexpr bool SYM = EPI <= kEpiSymAdd;
  const bool row = m < p.M;
  const int left = p.N - n;
  // A stored row is read up to its padding, so the padding is written too: that of a
  // symmetric matrix's upper rows by the mirrored tiles, from rows past M.
  if (EPI == kEpiUpdate ? !row || left <= 0 : n >= p.o.pad || !(row || (SYM && m < p.o.pad))) return;
  float v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = row ? p.zs * z[q] : 0.f;
    if (EPI != kEpiSym && row) v[q] = fmaf(p.cs, (float)x.h[q] + (float)x.l[q], v[q]);
  }
  if constexpr (EPI == kEpiUpdate) {
    T* w = static_cast<T*>(p.W) + ((int64_t)mat * p.M + m) * p.N + n;
    if (left >= 4) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = fmaf(-p.us, v[q], p.ws * Vec<T, 4>::get(x.w, q));
      Vec<T, 4>::put(w, v);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < left) {
          const float y[1] = {fmaf(-p.us, v[q], p.ws * Elt<T>::get(w + q))};
          Vec<T, 1>::put(w + q, y);
        }
    }
  } else {
    uint16_t* o = p.o.p + mat * p.o.step;
    if (row) put4(o + spot(p.o, m, n), v);
    if (SYM && mirror) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < left) put1(o + spot(p.o, n + q, m), v[q]);
    }
  }
}

// Tiles of a block and of a wave, and stages of k in LDS.
template <int BM_, int BN_, int WM_, int WN_, int ST_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, ST = ST_;
  static constexpr int NWN = BN / WN, NW = (BM / WM) * NWN, NT = NW * 64, MI = WM / 16, NI = WN / 16;
  static constexpr size_t kLds = (size_t)ST * (BM + BN) * 128;
};

// Waits until at most N loads of this wave are in flight.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <class TL, bool AKM, bool BKM, int EPI, class T>
__global__ void __launch_bounds__(TL::NT) k_muon_product(const MuonArgs p) {
  constexpr int BM = TL::BM, BN = TL::BN, MI = TL::MI, NI = TL::NI, NW = TL::NW, ST = TL::ST;
  constexpr int PL = 2, BK = 32;  // parts of a value, k of a stage
  // by rows of k: 32 values in two parts; with k as the row: 32 rows of the tile's columns in theirs
  typedef GTile<AKM ? BM : BM * PL, AKM ? 64 : BK, AKM, NW, false> TA;
  typedef GTile<BKM ? BN : BN * PL, BKM ? 64 : BK, BKM, NW, false> TB;
  constexpr int kStage = TA::kBytes + TB::kBytes, kLoads = TA::PER + TB::PER;
  static_assert((size_t)ST * kStage == TL::kLds && kLoads * (ST - 1) < 64, "the stages fit LDS and the counter");
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4, wm = wave / TL::NWN, wn = wave % TL::NWN;
  // a tile, or one of the parts of its k
  uint32_t tile = blockIdx.x, piece = 0, pieces = 1;
  if (tile >= p.full) {
    pieces = p.pieces;
    piece = (blockIdx.x - p.full) % pieces;
    tile = p.full + (blockIdx.x - p.full) / pieces;
  }
  uint32_t mat, im, in;
  tile_of<EPI>(p, tile, mat, im, in);
  const int m0 = (int)im * BM, n0 = (int)in * BN;
  const uint16_t *ap = p.a.p + mat * p.a.step, *bp = p.b.p + mat * p.b.step;
  const uint32_t whole = (uint32_t)(p.K + BK - 1) / BK;
  const int from = (int)(whole * piece / pieces), to = (int)(whole * (piece + 1) / pieces);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(g_lds_addr(lds));
  TA ta;
  TB tb;
  ta.init(GOperand<uint16_t>{ap, p.a.ld, p.a.rows, p.a.ld}, wave, lane, 0);
  tb.init(GOperand<uint16_t>{bp, p.b.ld, p.b.rows, p.b.ld}, wave, lane, 0);

  // (rows past the last and values past a row's padding read as zero)
  auto issue = [&](int t) {
    const uint32_t st = lds0 + (uint32_t)(t % ST) * kStage;
    const int64_t kv = (int64_t)t * 64, kr = (int64_t)t * BK;
    if constexpr (AKM) {
      ta.issue(ap + (int64_t)m0 * p.a.ld + kv, 2 * ((int64_t)(p.a.rows - m0) * p.a.ld - kv), p.a.ld - kv, st, wave);
    } else {
      ta.issue(ap + kr * p.a.ld + m0 * PL, 2 * ((p.a.rows - kr) * p.a.ld - m0 * PL), p.K - kr, st, wave);
    }
    if constexpr (BKM) {
      tb.issue(bp + (int64_t)n0 * p.b.ld + kv, 2 * ((int64_t)(p.b.rows - n0) * p.b.ld - kv), p.b.ld - kv, st + TA::kBytes, wave);
    } else {
      tb.issue(bp + kr * p.b.ld + n0 * PL, 2 * ((p.b.rows - kr) * p.b.ld - n0 * PL), p.K - kr, st + TA::kBytes, wave);
    }
  };

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int q = 0; q < ST - 1; ++q)
    if (from + q < to) issue(from + q);
  for (int t = from; t < to; ++t) {
    // this wave's share of the stage is in LDS, later stages may be under way
    if (to - t >= ST - 1) {
      wait_loads<kLoads*(ST - 2)>();
    } else {
      wait_loads<0>();
    }
    __syncthreads();
    if (t + ST - 1 < to) issue(t + ST - 1);
    const char* sa = lds + (t % ST) * kStage;
    const char* sb = sa + TA::kBytes;
    // fragment (i, part)
    auto fa_of = [&](int i, int h) { return AKM ? TA::frag(sa, i, h, c, g) : TA::frag(sa, (i >> 1) * 4 + (i & 1) + 2 * h, 0, c, g); };
    auto fb_of = [&](int i, int h) { return BKM ? TB::frag(sb, i, h, c, g) : TB::frag(sb, (i >> 1) * 4 + (i & 1) + 2 * h, 0, c, g); };
    uint4 fa[2][MI], fb[2][NI];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < NI; ++j) fb[h][j] = fb_of(wn * NI + j, h);
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[h][i] = fa_of(wm * MI + i, h);
    }
#pragma unroll
    for (int h = 0; h < 3; ++h)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mfma_f16(fb[h == 1][j], fa[h == 2][i], acc[i][j]);
  }

  if (pieces > 1) {
    float* mine = p.part + (int64_t)(blockIdx.x - p.full) * BM * BN + threadIdx.x * 4;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) *reinterpret_cast<f32x4*>(mine + (i * NI + j) * TL::NT * 4) = acc[i][j];
    return;
  }
  // lane (c, g) holds columns 16 j + 4 g .. + 3 of row 16 i + c
  const int mr = m0 + wm * TL::WM + c, nc = n0 + wn * TL::WN + 4 * g;
  Beside<EPI, T> x[2][NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) x[0][j].load(p, mat, mr, nc + 16 * j);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    if (i + 1 < MI)
#pragma unroll
      for (int j = 0; j < NI; ++j) x[(i + 1) & 1][j].load(p, mat, mr + 16 * (i + 1), nc + 16 * j);
#pragma unroll
    for (int j = 0; j < NI; ++j) finish<EPI, T>(p, mat, mr + 16 * i, nc + 16 * j, im != in, acc[i][j], x[i & 1][j]);
  }
}

// Tiles whose k was cut: their parts added in order, then the epilogue.  A block has
// one of the MI NI groups of 16 x 16 of each of a tile's waves.
template <class TL, int EPI, class T>
__global__ void __launch_bounds__(TL::NT) k_muon_join(const MuonArgs p) {
  constexpr int G = TL::MI * TL::NI;
  const uint32_t cut = blockIdx.x / G, ij = blockIdx.x - cut * G;
  uint32_t mat, im, in;
  tile_of<EPI>(p, p.full + cut, mat, im, in);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4, i = (int)ij / TL::NI, j = (int)ij % TL::NI;
  const float* all = p.part + (int64_t)cut * p.pieces * TL::BM * TL::BN + (int64_t)ij * TL::NT * 4 + threadIdx.x * 4;
  const int m = (int)im * TL::BM + (wave / TL::NWN) * TL::WM + 16 * i + c;
  const int n = (int)in * TL::BN + (wave % TL::NWN) * TL::WN + 16 * j + 4 * g;
  Beside<EPI, T> x;
  x.load(p, mat, m, n);
  f32x4 z{0.f, 0.f, 0.f, 0.f};
  for (int q0 = 0; q0 < p.pieces; q0 += 8) {
    f32x4 y[8];
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q0 + q < p.pieces) y[q] = *reinterpret_cast<const f32x4*>(all + (int64_t)(q0 + q) * TL::BM * TL::BN);
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q0 + q < p.pieces)
#pragma unroll
        for (int v = 0; v < 4; ++v) z[v] += y[q][v];
  }
  finish<EPI, T>(p, mat, m, n, im != in, z, x);
}

// ---- momentum, norm, first X ------------------------------------------------------
constexpr int kNormBlocks = 2048;  // blocks of a matrix at most

// M = mu M + G and the blocks' sums of U^2: four values at a time, the last ones
// (and all of a matrix whose four would reach into the next) one by one.
template <class T>
__global__ void __launch_bounds__(256)
    k_muon_momentum(const T* __restrict__ G, float* __restrict__ M, int64_t n, float mu, int nesterov, double* __restrict__ part) {
  __shared__ double sh[256];
  const T* g = G + (int64_t)blockIdx.y * n;
  float* m = M + (int64_t)blockIdx.y * n;
  double s = 0;
  const int64_t step = (int64_t)gridDim.x * 1024;
  for (int64_t i0 = (int64_t)blockIdx.x * 1024 + threadIdx.x * 4; i0 < n; i0 += 4 * step) {
    typename Vec<T, 4>::raw a[4];
    typename Vec<float, 4>::raw b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + k * step + 4 <= n) {
        a[k] = Vec<T, 4>::load(g + i0 + k * step);
        b[k] = Vec<float, 4>::load(m + i0 + k * step);
      }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t i = i0 + k * step;
      if (i + 4 <= n) {
        float v[4];
        double w = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float x = Vec<T, 4>::get(a[k], q);
          v[q] = fmaf(mu, b[k][q], x);
          const double u = nesterov ? fmaf(mu, v[q], x) : v[q];
          w += u * u;
        }
        s += w;
        Vec<float, 4>::put(m + i, v);
      } else {
        for (int64_t q = i; q < n; ++q) {
          const float x = Elt<T>::get(g + q), v = fmaf(mu, m[q], x);
          m[q] = v;
          const double u = nesterov ? fmaf(mu, v, x) : v;
          s += u * u;
        }
      }
    }
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  for (int o = 128; o > 0; o /= 2) {
    if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sh[0];
}

// 1 / max(size, eps) as f 2^e (so that neither it nor a scaled value leaves float32's
// range); NaN if the size is not finite.
struct Inverse {
  float f;
  int e;
};
__device__ __forceinline__ Inverse inverse_of(double size, float eps) {
  int e;
  const double f = frexp(1.0 / (size > (double)eps ? size : (double)eps), &e);
  return std::isfinite(size) ? Inverse{(float)f, e} : Inverse{__builtin_nanf(""), 0};
}
__device__ __forceinline__ float scaled(float u, const Inverse& i, int more) {
  return __builtin_amdgcn_ldexpf(u * i.f, i.e + more);
}

// X = U / max(|U|, eps) in its parts, or with steps = 0 the update of W.
template <class T, bool UPDATE>
__global__ void __launch_bounds__(256)
    k_muon_first(const T* __restrict__ G, const float* __restrict__ M, int32_t rows, int32_t cols, float mu, int nesterov,
                 const double* __restrict__ part, int parts, float eps, Stored o, T* __restrict__ W, float ws, float us) {
  __shared__ double sh[256];
  const int64_t mat = blockIdx.y, base = mat * rows * cols;
  {
    double s = 0;
    for (int q = threadIdx.x; q < parts; q += 256) s += part[mat * parts + q];
    sh[threadIdx.x] = s;
  }
  __syncthreads();
  for (int q = 128; q > 0; q /= 2) {
    if ((int)threadIdx.x < q) sh[threadIdx.x] += sh[threadIdx.x + q];
    __syncthreads();
  }
  const Inverse inv = inverse_of(sqrt(sh[0]), eps);
  const int per = o.pad / 4;
  const int64_t n = (int64_t)rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / per), c = (int)(i - (int64_t)r * per) * 4;
    const int64_t at = base + (int64_t)r * cols + c;
    float v[4] = {0.f, 0.f, 0.f, 0.f}, g[4], m[4], w[4];
    const int left = cols - c;
    if (left >= 4) {
      const auto a = Vec<T, 4>::load(G + at);
      const auto b = Vec<float, 4>::load(M + at);
      if constexpr (UPDATE) {
        const auto d = Vec<T, 4>::load(W + at);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = Vec<T, 4>::get(d, q);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) g[q] = Vec<T, 4>::get(a, q), m[q] = b[q];
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        g[q] = q < left ? Elt<T>::get(G + at + q) : 0.f;
        m[q] = q < left ? M[at + q] : 0.f;
        if (UPDATE) w[q] = q < left ? Elt<T>::get(W + at + q) : 0.f;
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q >= left) break;
      const float x = scaled(nesterov ? fmaf(mu, m[q], g[q]) : m[q], inv, UPDATE ? 0 : kXe);
      v[q] = UPDATE ? fmaf(-us, x, ws * w[q]) : x;
    }
    if constexpr (!UPDATE) {
      put4(o.p + mat * o.step + spot(o, r, c), v);
    } else if (left >= 4) {
      Vec<T, 4>::put(W + at, v);
    } else {
      for (int q = 0; q < left; ++q) {
        const float y[1] = {v[q]};
        Vec<T, 1>::put(W + at + q, y);
      }
    }
  }
}

// ---- small matrices -----------------------------------------------------------------
// A matrix whose smaller side is at most MP and whose X and A fit LDS: one block does
// the whole update.  X [MP][pad of the larger side] and A [MP][MP] lie in LDS in
// panels of 128-byte rows (the stored rows' order), the 16-byte chunk ch of row r at
// ch ^ (r & 7).  A panel is a tile by rows of k (the Gram product, A A, B), or with
// transposing reads one with k as the row (B X).  A tall matrix is worked on as its
// transpose.  A product's sums stay in registers until all waves have read, so A A
// overwrites A, and B X overwrites X.
struct SmallArgs {
  const void* G;
  float* M;
  void* W;
  int32_t rows, cols;   // as the caller has them
  int32_t m, n, panels; // the smaller side, the larger, panels of X
  int32_t steps, nesterov;
  float mu, eps, ws, us;
};

constexpr int kSmallWaves = 16;
constexpr size_t kSmallStatic = (size_t)kSmallWaves * 64 * sizeof(double);  // the norm's sums
constexpr size_t kSmallLds = 160 * 1024 - kSmallStatic;                    // X and A at most
constexpr int kFlight = 4;  // times four values of a thread in flight

// fragment of rows 16 i + c of a panel, k = 32 kb + 8 g ..
__device__ __forceinline__ uint4 panel_rows(const char* panel, int i, int kb, int c, int g) {
  return *reinterpret_cast<const uint4*>(panel + (16 * i + c) * 128 + (((4 * kb + g) ^ (c & 7)) * 16));
}
// fragment of columns 16 j + c of a panel (16-bit values of its rows), k = rows 32 kb + 8 g ..
__device__ __forceinline__ uint4 panel_cols(const char* panel, int j, int kb, int c, int g) {
  typedef __attribute__((address_space(3))) g_s16x4* lds_ptr;
  const int r = 32 * kb + 8 * g + (c >> 2), ch = 2 * j + ((c & 3) >> 1);
  const char* a = panel + r * 128 + ((ch ^ (r & 7)) * 16) + (c & 1) * 8;
  const char* b = panel + (r + 4) * 128 + ((ch ^ ((r + 4) & 7)) * 16) + (c & 1) * 8;
  const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)a));
  const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)b));
  return uint4{x.x, x.y, y.x, y.y};
}
// the high part of value (r, col) of panels of MP rows
template <int MP>
__device__ __forceinline__ uint16_t* panel_at(char* panels, int r, int col) {
  const int panel = col >> 5, v = col & 31;
  return reinterpret_cast<uint16_t*>(panels + panel * MP * 128 + r * 128 + (((v >> 3) ^ (r & 7)) * 16)) + (v & 7);
}
// (the low part's chunk is four from the high part's, before the exchange by r & 7)
template <int MP>
__device__ __forceinline__ void panel_put4(char* panels, int r, int col, const float (&v)[4]) {
  f16x4 h, l;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h[q] = (_Float16)v[q];
    l[q] = (_Float16)(v[q] - (float)h[q]);
  }
  uint16_t* p = panel_at<MP>(panels, r, col);
  *reinterpret_cast<f16x4*>(p) = h;
  *reinterpret_cast<f16x4*>(reinterpret_cast<uint16_t*>(reinterpret_cast<uintptr_t>(p) ^ 64)) = l;
}
template <int MP>
__device__ __forceinline__ void panel_get4(const char* panels, int r, int col, float (&v)[4]) {
  const uint16_t* p = panel_at<MP>(const_cast<char*>(panels), r, col);
  const f16x4 h = *reinterpret_cast<const f16x4*>(p);
  const f16x4 l = *reinterpret_cast<const f16x4*>(reinterpret_cast<const uint16_t*>(reinterpret_cast<uintptr_t>(p) ^ 64));
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = (float)h[q] + (float)l[q];
}

// One stage of k (a panel's 128-byte rows) into acc: hi hi and the cross products.
template <int MI, int NI, class FA, class FB>
__device__ __forceinline__ void stage(f32x4 (&acc)[MI][NI], FA fa_of, FB fb_of) {
  uint4 fa[2][MI], fb[2][NI];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int j = 0; j < NI; ++j) fb[h][j] = fb_of(j, h);
#pragma unroll
    for (int i = 0; i < MI; ++i) fa[h][i] = fa_of(i, h);
  }
#pragma unroll
  for (int h = 0; h < 3; ++h)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mfma_f16(fb[h == 1][j], fa[h == 2][i], acc[i][j]);
}
template <int MI, int NI>
__device__ __forceinline__ void clear(f32x4 (&acc)[MI][NI]) {
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

template <class T, int MP>
__global__ void __launch_bounds__(kSmallWaves * 64) k_muon_small(const SmallArgs p) {
  constexpr int CP = 32;                           // columns of a panel
  constexpr int NT = kSmallWaves * 64, kPanel = MP * 128, AP = MP / CP;
  constexpr int WR = MP / 16 < 4 ? MP / 16 : 4, WC = WR;  // waves of A
  constexpr int MI = MP / 16 / WR, NI = MP / 16 / WC;
  constexpr int XR = MP / 32, XI = MP / 16 / XR;  // row parts of a panel of X, their 16-row blocks
  constexpr int XJ = CP / 16;
  extern __shared__ __align__(1024) char lds[];
  __shared__ double sh[NT];
  static_assert(sizeof(sh) == kSmallStatic, "the LDS beside the panels");
  char *xs = lds, *as = lds + p.panels * kPanel;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const int64_t size = (int64_t)p.rows * p.cols, base = blockIdx.x * size;
  const T* G = static_cast<const T*>(p.G) + base;
  float* M = p.M + base;
  T* W = static_cast<T*>(p.W) + base;
  const bool tall = p.rows > p.cols;

  // four values a thread, kFlight times in flight; the matrix's last ones by one thread
  const int n4 = (int)(size / 4) * 4, left = (int)size - n4;
  const auto pass = [&](auto f) {
    for (int i0 = threadIdx.x * 4; i0 < n4; i0 += NT * 4 * kFlight) {
      typename Vec<T, 4>::raw x[kFlight];
      typename Vec<float, 4>::raw m[kFlight];
#pragma unroll
      for (int k = 0; k < kFlight; ++k)
        if (i0 + k * NT * 4 < n4) {
          x[k] = Vec<T, 4>::load(G + i0 + k * NT * 4);
          m[k] = Vec<float, 4>::load(M + i0 + k * NT * 4);
        }
#pragma unroll
      for (int k = 0; k < kFlight; ++k)
        if (i0 + k * NT * 4 < n4) {
          const float xs4[4] = {Vec<T, 4>::get(x[k], 0), Vec<T, 4>::get(x[k], 1), Vec<T, 4>::get(x[k], 2), Vec<T, 4>::get(x[k], 3)};
          const float ms4[4] = {m[k][0], m[k][1], m[k][2], m[k][3]};
          f(i0 + k * NT * 4, xs4, ms4, 4);
        }
    }
    if ((int)threadIdx.x < left) {
      const float x1[4] = {Elt<T>::get(G + n4 + threadIdx.x), 0.f, 0.f, 0.f}, m1[4] = {M[n4 + threadIdx.x], 0.f, 0.f, 0.f};
      f(n4 + (int)threadIdx.x, x1, m1, 1);
    }
  };
  double s = 0;
  pass([&](int i, const float (&x)[4], const float (&m)[4], int n) {
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = fmaf(p.mu, m[q], x[q]);
      const double u = p.nesterov ? fmaf(p.mu, v[q], x[q]) : v[q];
      if (q < n) s += u * u;
    }
    if (n == 4) {
      Vec<float, 4>::put(M + i, v);
    } else {
      M[i] = v[0];
    }
  });
  sh[threadIdx.x] = s;
  // (X's padding and rows past m are zero, and what no product writes of A's panels)
  for (int i = threadIdx.x; i < (p.panels + AP) * kPanel / 16; i += NT) reinterpret_cast<uint4*>(xs)[i] = uint4{0u, 0u, 0u, 0u};
  __syncthreads();
  for (int o = NT / 2; o > 0; o /= 2) {
    if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  const Inverse inv = inverse_of(sqrt(sh[0]), p.eps);
  // (a thread reads again what it wrote)
  pass([&](int i, const float (&x)[4], const float (&m)[4], int n) {
    int r = i / p.cols, q = i - r * p.cols;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k >= n) break;
      const float y = scaled(p.nesterov ? fmaf(p.mu, m[k], x[k]) : m[k], inv, kXe);
      uint16_t* o = panel_at<MP>(xs, tall ? q : r, tall ? r : q);
      const _Float16 h = (_Float16)y;
      *o = __builtin_bit_cast(uint16_t, h);
      *reinterpret_cast<uint16_t*>(reinterpret_cast<uintptr_t>(o) ^ 64) = __builtin_bit_cast(uint16_t, (_Float16)(y - (float)h));
      if (++q == p.cols) q = 0, ++r;
    }
  });
  __syncthreads();

  const int wr = wave / WC, wc = wave % WC;
  const bool mine = wave < WR * WC;
  const int units = p.panels * XR;
  for (int it = 0; it < p.steps; ++it) {
    f32x4 acc[MI][NI];
    // A = X X^T
    clear(acc);
    if (mine)
      for (int q = 0; q < p.panels; ++q) {
        const char* x = xs + q * kPanel;
        stage(acc, [&](int i, int h) { return panel_rows(x, wr * MI + i, h, c, g); },
                  [&](int j, int h) { return panel_rows(x, wc * NI + j, h, c, g); });
      }
    auto store = [&](float zs) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const int r = 16 * (wr * MI + i) + c, col = 16 * (wc * NI + j) + 4 * g;
          float v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = zs * acc[i][j][k];
          panel_put4<MP>(as, r, col, v);
        }
    };
    if (mine) store(pow2(kAe - 2 * kXe));
    __syncthreads();
    // B = q A + s A A, over A
    clear(acc);
    if (mine) {
#pragma unroll
      for (int q = 0; q < AP; ++q) {
        const char* x = as + q * kPanel;
        stage(acc, [&](int i, int h) { return panel_rows(x, wr * MI + i, h, c, g); },
                  [&](int j, int h) { return panel_rows(x, wc * NI + j, h, c, g); });
      }
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          float v[4];
          panel_get4<MP>(as, 16 * (wr * MI + i) + c, 16 * (wc * NI + j) + 4 * g, v);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            acc[i][j][k] = fmaf(kQ * pow2(kBe - kAe), v[k], kS * pow2(kBe - 2 * kAe) * acc[i][j][k]);
        }
    }
    __syncthreads();
    if (mine) store(1.f);
    __syncthreads();
    // X = p X + B X: a wave has a panel's columns, and of those 32 rows
    for (int u0 = 0; u0 < units; u0 += kSmallWaves) {
      const int u = u0 + wave, panel = u / XR, part = u - panel * XR;
      char* x = xs + panel * kPanel;
      f32x4 z[XI][XJ];
      clear(z);
      if (u < units) {
#pragma unroll
        for (int q = 0; q < MP / 32; ++q) {
          // rows of B: 32 of its columns in two parts
          const char* bq = as + q * kPanel;
          uint4 fa[2][XI], fb[2][XJ];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < XI; ++i) fa[h][i] = panel_rows(bq, part * XI + i, h, c, g);
#pragma unroll
            for (int j = 0; j < XJ; ++j) fb[h][j] = panel_cols(x, j + 2 * h, q, c, g);
          }
#pragma unroll
          for (int h = 0; h < 3; ++h)
#pragma unroll
            for (int i = 0; i < XI; ++i)
#pragma unroll
              for (int j = 0; j < XJ; ++j) z[i][j] = mfma_f16(fb[h == 1][j], fa[h == 2][i], z[i][j]);
        }
#pragma unroll
        for (int i = 0; i < XI; ++i)
#pragma unroll
          for (int j = 0; j < XJ; ++j) {
            float v[4];
            panel_get4<MP>(x, 16 * (part * XI + i) + c, 16 * j + 4 * g, v);
#pragma unroll
            for (int k = 0; k < 4; ++k) z[i][j][k] = fmaf(kP, v[k], pow2(-kBe) * z[i][j][k]);
          }
      }
      if (XR > 1) __syncthreads();  // (the other rows' wave of the panel has read it)
      if (u < units)
#pragma unroll
        for (int i = 0; i < XI; ++i)
#pragma unroll
          for (int j = 0; j < XJ; ++j) {
            const float v[4] = {z[i][j][0], z[i][j][1], z[i][j][2], z[i][j][3]};
            panel_put4<MP>(xs, 16 * (part * XI + i) + c, panel * CP + 16 * j + 4 * g, v);
          }
    }
    __syncthreads();
  }

  // W along X, in W's order (a lane's values of the last product lie in 16 rows: 13 us
  // more for 128 x 128 float32)
  const auto x_at = [&](int r, int q) {
    const uint16_t* o = panel_at<MP>(xs, tall ? q : r, tall ? r : q);
    return (float)__builtin_bit_cast(_Float16, *o) +
           (float)__builtin_bit_cast(_Float16, *reinterpret_cast<const uint16_t*>(reinterpret_cast<uintptr_t>(o) ^ 64));
  };
  for (int i0 = threadIdx.x * 4; i0 < n4; i0 += NT * 4 * kFlight) {
    typename Vec<T, 4>::raw w[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      if (i0 + k * NT * 4 < n4) w[k] = Vec<T, 4>::load(W + i0 + k * NT * 4);
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int i = i0 + k * NT * 4;
      if (i >= n4) break;
      int r = i / p.cols, q = i - r * p.cols;
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = fmaf(-p.us, x_at(r, q), p.ws * Vec<T, 4>::get(w[k], j));
        if (++q == p.cols) q = 0, ++r;
      }
      Vec<T, 4>::put(W + i, v);
    }
  }
  if ((int)threadIdx.x < left) {
    const int i = n4 + (int)threadIdx.x, r = i / p.cols;
    const float y[1] = {fmaf(-p.us, x_at(r, i - r * p.cols), p.ws * Elt<T>::get(W + i))};
    Vec<T, 1>::put(W + i, y);
  }
}

// ---- host ---------------------------------------------------------------------------
// Blocks of a launch's last round whose tiles are cut along k, and their parts.
constexpr int kParts = 512;       // blocks of parts at most
// Stages of k of a part at least (3 of 517 x 200 bfloat16: 133 us with 8, 139 with 16; 1024 x
// 1024 float32 265, 283, 335 with 24; 512 x 2048 184, 195, 219; 1024 x 5632 520, 517, 499).
constexpr int kLeastSteps = 8;

struct Bufs {
  double* part = nullptr;
  float* sums = nullptr;
  Stored x0{}, x1{}, a{}, b{};
  int parts = 0;
};

// The rows that a block holds a small matrix in, or 0; its LDS.
int small_of(const hg_muon_desc* A, size_t* bytes) {
  const int32_t m = std::min(A->rows, A->cols), n = std::max(A->rows, A->cols);
  if (A->steps == 0 || m > 128) return 0;
  const int mp = m <= 32 ? 32 : m <= 64 ? 64 : 128;
  const size_t panels = (size_t)(cdiv(n, 32) + mp / 32), need = panels * mp * 128;
  if (need > kSmallLds) return 0;
  *bytes = need;
  return mp;
}

template <class Mem>
Stored stored(const hg_muon_desc* A, int32_t rows, int32_t cols, bool memory, Mem& m) {
  Stored p{};
  p.rows = rows;
  p.cols = cols;
  p.pad = (cols + 31) / 32 * 32;
  p.ld = 2 * p.pad;
  p.step = (int64_t)rows * p.ld;
  if (memory) p.p = m.template take<uint16_t>(p.step * A->count);
  return p;
}

template <class Mem>
Bufs take(const hg_muon_desc* A, Mem& m) {
  Bufs b;
  size_t bytes = 0;
  if (small_of(A, &bytes)) return b;
  const int64_t n = (int64_t)A->rows * A->cols;
  const int32_t k = std::min(A->rows, A->cols);
  b.parts = (int)std::min<int64_t>(kNormBlocks, std::max<int64_t>(1, cdiv(n, 1024)));
  b.part = m.template take<double>((int64_t)A->count * b.parts);
  const bool any = A->steps > 0;
  b.sums = m.template take<float>(any ? (int64_t)kParts * 128 * 128 : 0);
  b.x0 = stored(A, A->rows, A->cols, any, m);
  b.x1 = stored(A, A->rows, A->cols, A->steps > 1, m);
  b.a = stored(A, k, k, any, m);
  b.b = stored(A, k, k, any, m);
  return b;
}

int check(const hg_muon_desc* A, const char* what) {
  if (!A) return fail(HG_ERR_ARG, "%s: null descriptor", what);
  if (A->count < 0 || A->rows < 1 || A->cols < 1)
    return fail(HG_ERR_ARG, "%s: %d matrices of %d x %d", what, A->count, A->rows, A->cols);
  if (A->dtype != HG_DTYPE_F32 && A->dtype != HG_DTYPE_BF16) return fail(HG_ERR_ARG, "%s: dtype %d", what, A->dtype);
  if (A->steps < 0 || A->steps > 32) return fail(HG_ERR_ARG, "%s: steps %d", what, A->steps);
  if (A->nesterov != 0 && A->nesterov != 1) return fail(HG_ERR_ARG, "%s: nesterov %d", what, A->nesterov);
  if (!std::isfinite(A->lr) || !std::isfinite(A->mu) || !std::isfinite(A->weight_decay) || !std::isfinite(A->scale) ||
      !(A->eps > 0.f) || !std::isfinite(A->eps))
    return fail(HG_ERR_ARG, "%s: lr=%g mu=%g weight_decay=%g scale=%g eps=%g", what, (double)A->lr, (double)A->mu,
                (double)A->weight_decay, (double)A->scale, (double)A->eps);
  if (A->rows > 1 << 15 || A->cols > 1 << 15 || (int64_t)A->rows * A->cols * A->count >= (int64_t)1 << 32 || A->count > 65535 ||
      cdiv(A->rows, 64) * cdiv(A->cols, 64) * A->count >= 1 << 22)
    return fail(HG_ERR_UNSUPPORTED, "%s: %d matrices of %d x %d", what, A->count, A->rows, A->cols);
  return HG_OK;
}

// Tiles of the last round may be cut along k.  Not those of the products with X, whose
// sums are larger than what the cut saves (1024 x 1024 float32 266 us, 294 with).
template <class TL, bool AKM, bool BKM, int EPI, class T>
int product(const char* name, MuonArgs a, int count, hipStream_t s) {
  constexpr bool CUT = EPI <= kEpiSymAdd;
  a.tiles_m = (a.M + TL::BM - 1) / TL::BM;
  a.tiles_n = (a.N + TL::BN - 1) / TL::BN;
  a.tiles = EPI <= kEpiSymAdd ? a.tiles_m * (a.tiles_m + 1) / 2 : a.tiles_m * a.tiles_n;
  constexpr auto kernel = k_muon_product<TL, AKM, BKM, EPI, T>;
  HG_TRY((allow_lds<kernel, TL::kLds>()));
  // one block a tile in whole rounds of the chip; the rest in parts, if that helps
  const int64_t tiles = (int64_t)a.tiles * count, slots = (int64_t)num_cus() * std::max<int64_t>(1, 160 * 1024 / (int64_t)TL::kLds);
  const int64_t rest = tiles % slots, steps = cdiv(a.K, 32);
  a.pieces = 1;
  if (CUT && rest)
    a.pieces = (int32_t)std::max<int64_t>(1, std::min(std::min<int64_t>(slots, kParts) / rest, steps / kLeastSteps));
  a.full = (uint32_t)(a.pieces > 1 ? tiles - rest : tiles);
  HG_LAUNCH(name, kernel, dim3((unsigned)(a.full + (tiles - a.full) * a.pieces)), dim3(TL::NT), TL::kLds, s, a);
  if constexpr (CUT) {
    if (a.pieces > 1)
      HG_LAUNCH("muon_join", (k_muon_join<TL, EPI, T>), dim3((unsigned)(rest * TL::MI * TL::NI)), dim3(TL::NT), 0, s, a);
  }
  return HG_OK;
}

typedef Tile<64, 64, 32, 32, 4> T64;
typedef Tile<64, 128, 32, 64, 2> T64x128;
typedef Tile<128, 128, 64, 64, 2> T128;
typedef Tile<256, 256, 128, 64, 2> T256;

// Symmetric products: tiles of 128 x 128 where there are many, or k is long, and they cover
// little more than tiles of 64 x 64, whose sums of cut tiles are smaller.  Whole updates with
// either for A, by tiles of 128 x 128 times k: 1024 x 4096 (36 x 4096) 427 us, 416 with 64 x 64;
// 1024 x 5120 491, 499; 4 of 1024 x 1024 (144 x 1024) 486, 463; 16 of 600 x 2400 (240 x 2400)
// 1.17 ms, 1.25; 2048 x 4096 (136 x 4096) 1.07 ms, 1.15.  Rows that fill no tile: 64 of 300 x
// 2000 (60% more covered) 1.41 ms, 1.49; 64 of 130 x 2000 (twice as much) 622 us, 572.
template <bool AKM, int EPI, class T>
int symmetric(const char* name, const MuonArgs& a, int count, hipStream_t s) {
  const auto tiles = [&](int64_t side) { return cdiv(a.M, side) * (cdiv(a.M, side) + 1) / 2; };
  const bool few128 = 4 * (double)tiles(128) <= 1.65 * (double)tiles(64);
  if (tiles(128) * count * a.K >= 160 * 1024 && few128) return product<T128, AKM, AKM, EPI, T>(name, a, count, s);
  return product<T64, AKM, AKM, EPI, T>(name, a, count, s);
}

// Products with X: of the tiles of which there are some for every CU, those that give the
// CU with the most of them the least work; the same work takes 5% longer in tiles of 128 x 128
// than of 256 x 256, 20% in 64 x 128.  A product of 2560 x 5120 (200 tiles of 256 x 256) takes 208
// us with them, 222 with 128 x 128, of 2304 x 5376 (189) 185 and 167; of 2500 x 2500 (400 of 128 x
// 128) 115 with them, 132 with 64 x 128, of 2048 x 2048 (256) 65 and 61; of 1536 x 1536 (288 of
// 64 x 128) 45 with them, 54 with 64 x 64, of 1024 x 2048 (256) 30 and 26.  Tiles that are partly
// empty, or leave CUs without one at the end: 3432 x 5264 (294 of 256 x 256, a whole update) 4.27
// ms, 3.54 with 128 x 128; 4 of 1100 x 5000 203 us, 171; 64 of 300 x 2000 164 us with 128 x 128,
// 154 with 64 x 128.
template <bool BKM, int EPI, class T>
int apply(const char* name, const MuonArgs& a, int count, hipStream_t s) {
  const int64_t cus = num_cus();
  const auto tiles = [&](int bm, int bn) { return cdiv(a.M, bm) * cdiv(a.N, bn) * count; };
  const auto most = [&](int bm, int bn, int64_t least, double slow) {
    return tiles(bm, bn) < least ? INFINITY : slow * (double)(cdiv(tiles(bm, bn), cus) * bm * bn);
  };
  const double w256 = most(256, 256, 192, 1.0), w128 = most(128, 128, 385, 1.05), w64 = most(64, 128, 257, 1.2);
  if (w256 <= std::min(w128, w64) && w256 < INFINITY) return product<T256, true, BKM, EPI, T>(name, a, count, s);
  if (w128 <= w64 && w128 < INFINITY) return product<T128, true, BKM, EPI, T>(name, a, count, s);
  if (w64 < INFINITY) return product<T64x128, true, BKM, EPI, T>(name, a, count, s);
  return product<T64, true, BKM, EPI, T>(name, a, count, s);
}

template <bool TALL, class TW>
int steps(const hg_muon_desc* A, const Bufs& b, void* W, hipStream_t s) {
  Stored x = b.x0, next = b.x1;
  const int32_t k = std::min(A->rows, A->cols), len = std::max(A->rows, A->cols);
  for (int i = 0; i < A->steps; ++i) {
    MuonArgs g{};
    g.part = b.sums;
    g.a = g.b = x;
    g.o = b.a;
    g.M = g.N = k;
    g.K = len;
    g.zs = pow2(kAe - 2 * kXe);
    HG_TRY((symmetric<!TALL, kEpiSym, TW>("muon_gram", g, A->count, s)));
    g.a = g.b = g.c = b.a;
    g.o = b.b;
    g.K = k;
    g.zs = kS * pow2(kBe - 2 * kAe);
    g.cs = kQ * pow2(kBe - kAe);
    HG_TRY((symmetric<true, kEpiSymAdd, TW>("muon_square", g, A->count, s)));
    g.a = TALL ? x : b.b;
    g.b = TALL ? b.b : x;
    g.c = x;
    g.o = next;
    g.M = A->rows;
    g.N = A->cols;
    g.K = k;
    g.zs = pow2(-kBe);
    g.cs = kP;
    if (i + 1 < A->steps) {
      HG_TRY((apply<TALL, kEpiAdd, TW>("muon_apply", g, A->count, s)));
      std::swap(x, next);
    } else {
      g.W = W;
      g.ws = 1.f - A->lr * A->weight_decay;
      g.us = A->lr * A->scale * pow2(-kXe);
      HG_TRY((apply<TALL, kEpiUpdate, TW>("muon_update", g, A->count, s)));
    }
  }
  return HG_OK;
}

template <class T, int MP>
int small(const hg_muon_desc* A, size_t bytes, T* W, const T* G, float* M, hipStream_t s) {
  SmallArgs a{};
  a.G = G;
  a.M = M;
  a.W = W;
  a.rows = A->rows;
  a.cols = A->cols;
  a.m = std::min(A->rows, A->cols);
  a.n = std::max(A->rows, A->cols);
  a.panels = (int32_t)cdiv(a.n, 32);
  a.steps = A->steps;
  a.nesterov = A->nesterov;
  a.mu = A->mu;
  a.eps = A->eps;
  a.ws = 1.f - A->lr * A->weight_decay;
  a.us = A->lr * A->scale * pow2(-kXe);
  constexpr auto kernel = k_muon_small<T, MP>;
  HG_TRY((allow_lds<kernel, kSmallLds, kSmallStatic>()));
  HG_LAUNCH("muon_small", kernel, dim3((unsigned)A->count), dim3(kSmallWaves * 64), bytes, s, a);
  return HG_OK;
}

template <class T>
int run(const hg_muon_desc* A, const Bufs& b, T* W, const T* G, float* M, hipStream_t s) {
  size_t bytes = 0;
  switch (small_of(A, &bytes)) {
    case 32: return small<T, 32>(A, bytes, W, G, M, s);
    case 64: return small<T, 64>(A, bytes, W, G, M, s);
    case 128: return small<T, 128>(A, bytes, W, G, M, s);
    default: break;
  }
  const int64_t n = (int64_t)A->rows * A->cols;
  const dim3 grid((unsigned)b.parts, (unsigned)A->count);
  HG_LAUNCH("muon_momentum", k_muon_momentum<T>, grid, dim3(256), 0, s, G, M, n, A->mu, A->nesterov, b.part);
  if (A->steps == 0) {
    HG_LAUNCH("muon_first", (k_muon_first<T, true>), grid, dim3(256), 0, s, G, M, A->rows, A->cols, A->mu, A->nesterov,
              b.part, b.parts, A->eps, b.x0, W, 1.f - A->lr * A->weight_decay, A->lr * A->scale);
    return HG_OK;
  }
  HG_LAUNCH("muon_first", (k_muon_first<T, false>), grid, dim3(256), 0, s, G, M, A->rows, A->cols, A->mu, A->nesterov, b.part,
            b.parts, A->eps, b.x0, W, 0.f, 0.f);
  return A->rows > A->cols ? steps<true, T>(A, b, W, s) : steps<false, T>(A, b, W, s);
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" size_t hg_muon_workspace_size(const hg_muon_desc* A) {
  if (check(A, "workspace size") != HG_OK || A->count == 0) return 0;
  Sizer m;
  take(A, m);
  return m.used;
}

extern "C" int hg_muon_step(const hg_muon_desc* A, void* W, const void* G, float* M, void* ws, size_t ws_bytes, void* stream) {
  const char* what = "hg_muon_step";
  HG_TRY(check(A, what));
  if (A->count == 0) return HG_OK;
  if (!W || !G || !M) return fail(HG_ERR_ARG, "%s: null pointer", what);
  const size_t n = (size_t)A->count * A->rows * A->cols, e = A->dtype == HG_DTYPE_F32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(W) | reinterpret_cast<uintptr_t>(G)) % e || reinterpret_cast<uintptr_t>(M) % 4)
    return fail(HG_ERR_ARG, "%s: a matrix is not aligned to its values", what);
  if (ranges_meet(W, n * e, G, n * e) || ranges_meet(W, n * e, M, n * 4) || ranges_meet(G, n * e, M, n * 4))
    return fail(HG_ERR_ARG, "%s: the matrices, their gradients and momenta overlap", what);
  Sizer need;
  take(A, need);
  HG_TRY(check_workspace(what, ws, ws_bytes, need.used));
  Arena m(ws, ws_bytes);
  const Bufs b = take(A, m);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return A->dtype == HG_DTYPE_F32
             ? run(A, b, static_cast<float*>(W), static_cast<const float*>(G), M, s)
             : run(A, b, static_cast<bf16_t*>(W), static_cast<const bf16_t*>(G), M, s);
}
