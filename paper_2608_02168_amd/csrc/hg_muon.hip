// One update of matrices along their orthogonalised momentum.
//
//   M = mu M + G,  U = G + mu M or M,  X = U / max(|U|, eps)
//   `steps` times:  A = X X^T,  B = q A + s A A,  X = p X + B X
//   W = (1 - lr wd) W - lr scale X
// (tall matrices: A = X^T X, X = p X + X B), (p, q, s) = (3.4445, -4.7750, 2.0315):
// singular values go through x (p + q x^2 + s x^4), which keeps [0, 1.21] in
// [0, 1.21] and takes small ones up by p a step.
//
// X, A and B are held in fp16 parts: the high part, and for float32 matrices what
// its rounding left (a float32 product is then hi hi + hi lo + lo hi, as in the
// row transforms).  Since no entry of X exceeds 1.21, of A 1.47 and of B 2.81,
// fixed powers of two take them to the top of fp16's range, exactly; a high part
// alone is off by 2^-12 of an entry down to 2^-28.  Sums are float32.
//
// Each product runs on the fp16 MFMA in tiles, with the tile loads of the linear
// map's products (hg_gemm.h): X is read as it lies, by rows or with k as the row
// index.  A and A A are symmetric: only tiles on and below the diagonal are
// formed, and written twice.  The sums q A + s A A and p X + B X and the update of
// W are the products' epilogues, so a step is three launches.
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

// One stored matrix [rows][ld] (ld a multiple of 8; columns past cols are zero), a
// plane or two of them, `step` values from one matrix of the call to the next.
struct Planes {
  uint16_t* p;
  int64_t step, lo;
  int32_t rows, cols, ld;
};

struct MuonArgs {
  Planes a, b;          // operands
  Planes c;             // what the epilogue adds: A for B, X for the next X
  Planes o;             // what it writes
  void* W;              // or the update of W [count][M][N]
  int32_t M, N, K;      // of the product
  int32_t tiles_m, tiles_n, tiles;  // tiles of one matrix
  float zs, cs;         // out = zs z + cs c
  float ws, us;         // W = ws W - us (zs z + cs c)
};

enum { kEpiSym = 0, kEpiSymAdd = 1, kEpiAdd = 2, kEpiUpdate = 3 };

// fp16 parts of four values; the low parts only with LO.
template <bool LO>
__device__ __forceinline__ void put4(const Planes& o, int64_t at, int left, const float (&v)[4]) {
  f16x4 h, l;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h[q] = (_Float16)v[q];
    l[q] = (_Float16)(v[q] - (float)h[q]);
  }
  if (left >= 4) {
    *reinterpret_cast<f16x4*>(o.p + at) = h;
    if (LO) *reinterpret_cast<f16x4*>(o.p + o.lo + at) = l;
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < left) {
        o.p[at + q] = __builtin_bit_cast(uint16_t, h[q]);
        if (LO) o.p[o.lo + at + q] = __builtin_bit_cast(uint16_t, l[q]);
      }
  }
}
template <bool LO>
__device__ __forceinline__ void get4(const Planes& c, int64_t at, float (&v)[4]) {
  const f16x4 h = *reinterpret_cast<const f16x4*>(c.p + at);
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = (float)h[q];
  if (LO) {
    const f16x4 l = *reinterpret_cast<const f16x4*>(c.p + c.lo + at);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += (float)l[q];
  }
}

// Tile (row, column) of tile id of the lower triangle.
__device__ __forceinline__ void tri_of(uint32_t id, uint32_t& im, uint32_t& in) {
  uint32_t i = (uint32_t)((sqrtf(8.f * (float)id + 1.f) - 1.f) * 0.5f);
  while ((i + 1) * (i + 2) / 2 <= id) ++i;
  while (i * (i + 1) / 2 > id) --i;
  im = i;
  in = id - i * (i + 1) / 2;
}

template <bool AKM, bool BKM, int BM, int BN, int WM, int WN, bool LO, int EPI, class TW>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64) k_muon_product(const MuonArgs p) {
  constexpr int BK = 64, NWN = BN / WN, NW = (BM / WM) * NWN, MI = WM / 16, NI = WN / 16, PL = LO ? 2 : 1;
  typedef GTile<BM, BK, AKM, NW, false> TA;
  typedef GTile<BN, BK, BKM, NW, false> TB;
  constexpr int kStage = PL * (TA::kBytes + TB::kBytes);
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4, wm = wave / NWN, wn = wave % NWN;
  const uint32_t mat = blockIdx.x / (uint32_t)p.tiles, id = blockIdx.x - mat * (uint32_t)p.tiles;
  constexpr bool SYM = EPI == kEpiSym || EPI == kEpiSymAdd;
  uint32_t im, in;
  if constexpr (SYM) {
    tri_of(id, im, in);
  } else {
    g_tile_of(id, p.tiles_m, p.tiles_n, 8, im, in);
  }
  const int m0 = (int)im * BM, n0 = (int)in * BN;
  const uint16_t *ap = p.a.p + mat * p.a.step, *bp = p.b.p + mat * p.b.step;
  const int steps = (p.K + BK - 1) / BK;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(g_lds_addr(lds));
  TA ta;
  TB tb;
  ta.init(GOperand<uint16_t>{ap, p.a.ld, p.a.rows, p.a.cols}, wave, lane, 0);
  tb.init(GOperand<uint16_t>{bp, p.b.ld, p.b.rows, p.b.cols}, wave, lane, 0);

  // (a stored row ends at ld, with zeros from cols on)
  auto issue = [&](int t) {
    const int64_t k0 = (int64_t)t * BK, kl = p.K - k0;
    uint32_t st = lds0 + (t & 1) * kStage;
#pragma unroll
    for (int q = 0; q < PL; ++q) {
      const uint16_t* s = ap + q * p.a.lo;
      if constexpr (AKM) {
        ta.issue(s + (int64_t)m0 * p.a.ld + k0, 2 * ((int64_t)(p.a.rows - m0) * p.a.ld - k0), kl, st, wave);
      } else {
        ta.issue(s + k0 * p.a.ld + m0, 2 * (kl * p.a.ld - m0), kl, st, wave);
      }
      st += TA::kBytes;
    }
#pragma unroll
    for (int q = 0; q < PL; ++q) {
      const uint16_t* s = bp + q * p.b.lo;
      if constexpr (BKM) {
        tb.issue(s + (int64_t)n0 * p.b.ld + k0, 2 * ((int64_t)(p.b.rows - n0) * p.b.ld - k0), kl, st, wave);
      } else {
        tb.issue(s + k0 * p.b.ld + n0, 2 * (kl * p.b.ld - n0), kl, st, wave);
      }
      st += TB::kBytes;
    }
  };

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  issue(0);
  for (int t = 0; t < steps; ++t) {
    g_wait_loads();  // this wave's share of the step is in LDS
    __syncthreads();
    if (t + 1 < steps) issue(t + 1);
    const char* sa = lds + (t & 1) * kStage;
    const char* sb = sa + PL * TA::kBytes;
#pragma unroll
    for (int kb = 0; kb < BK / 32; ++kb) {
      uint4 fa[PL][MI], fb[PL][NI];
#pragma unroll
      for (int q = 0; q < PL; ++q) {
#pragma unroll
        for (int j = 0; j < NI; ++j) fb[q][j] = TB::frag(sb + q * TB::kBytes, wn * NI + j, kb, c, g);
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[q][i] = TA::frag(sa + q * TA::kBytes, wm * MI + i, kb, c, g);
      }
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          if constexpr (LO) {
            acc[i][j] = mfma_f16(fb[0][j], fa[1][i], acc[i][j]);
            acc[i][j] = mfma_f16(fb[1][j], fa[0][i], acc[i][j]);
          }
          acc[i][j] = mfma_f16(fb[0][j], fa[0][i], acc[i][j]);
        }
    }
  }

  // lane (c, g) holds columns 16 j + 4 g .. + 3 of row 16 i + c
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int m = m0 + wm * WM + 16 * i + c;
    const bool row = m < p.M;
    // (a symmetric matrix's columns from M to ld are zeros that its mirrored tiles write)
    if (!row && !(SYM && m < p.o.ld)) continue;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + wn * WN + 16 * j + 4 * g, left = p.N - n;
      // (the padding of a written row is written too: a row is read up to ld)
      if (EPI == kEpiUpdate ? left <= 0 : n >= p.o.ld) continue;
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = row ? p.zs * acc[i][j][q] : 0.f;
      if constexpr (EPI != kEpiSym) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};  // (within the row: ld is a multiple of 8)
        if (row) get4<LO>(p.c, mat * p.c.step + (int64_t)m * p.c.ld + n, x);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = fmaf(p.cs, x[q], v[q]);
      }
      if constexpr (EPI == kEpiUpdate) {
        TW* w = static_cast<TW*>(p.W) + ((int64_t)mat * p.M + m) * p.N + n;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < left) {
            const float y = fmaf(-p.us, v[q], p.ws * Elt<TW>::get(w + q));
            if constexpr (sizeof(TW) == 4) {
              w[q] = y;
            } else {
              w[q] = f2bf(y);
            }
          }
      } else {
        // (columns from N to ld are zero: the operands' columns there are)
        if (row) put4<LO>(p.o, mat * p.o.step + (int64_t)m * p.o.ld + n, p.o.ld - n, v);
      }
      if constexpr (SYM) {
        if (im != in) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q < left) {
              const float s[4] = {v[q], 0.f, 0.f, 0.f};
              put4<LO>(p.o, mat * p.o.step + (int64_t)(n + q) * p.o.ld + m, 1, s);
            }
        }
      }
    }
  }
}

// ---- momentum, norm, first X ------------------------------------------------------
constexpr int kNormBlocks = 256;  // blocks of a matrix at most

// Four values from at on of n (fewer at the end).
template <class T>
__device__ __forceinline__ f32x4 take4(const T* p, int64_t left) {
  if (left >= 4) return Elt<T>::load4(p);
  f32x4 v{0.f, 0.f, 0.f, 0.f};
  for (int q = 0; q < left; ++q) v[q] = Elt<T>::get(p + q);
  return v;
}

// M = mu M + G and the blocks' sums of U^2.
template <class T>
__global__ void __launch_bounds__(256)
    k_muon_momentum(const T* __restrict__ G, float* __restrict__ M, int64_t n, float mu, int nesterov, double* __restrict__ part) {
  __shared__ double sh[256];
  const int64_t base = (int64_t)blockIdx.y * n;
  double s = 0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const float g = Elt<T>::get(G + base + i), m = fmaf(mu, M[base + i], g);
    M[base + i] = m;
    const double u = nesterov ? fmaf(mu, m, g) : m;
    s += u * u;
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  for (int o = 128; o > 0; o /= 2) {
    if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sh[0];
}

// X = U / max(|U|, eps) in its parts, or with steps = 0 the update of W.
template <class T, bool LO, bool UPDATE>
__global__ void __launch_bounds__(256)
    k_muon_first(const T* __restrict__ G, const float* __restrict__ M, int32_t rows, int32_t cols, float mu, int nesterov,
                 const double* __restrict__ part, int parts, float eps, Planes o, T* __restrict__ W, float ws, float us) {
  __shared__ double sh[kNormBlocks];
  const int64_t mat = blockIdx.y, base = mat * rows * cols;
  sh[threadIdx.x] = (int)threadIdx.x < parts ? part[mat * parts + threadIdx.x] : 0.0;
  __syncthreads();
  for (int q = kNormBlocks / 2; q > 0; q /= 2) {
    if ((int)threadIdx.x < q) sh[threadIdx.x] += sh[threadIdx.x + q];
    __syncthreads();
  }
  const double size = sqrt(sh[0]);
  const double inv = std::isfinite(size) ? 1.0 / (size > (double)eps ? size : (double)eps) : (double)__builtin_nanf("");
  const int per = o.ld / 4;
  const int64_t n = (int64_t)rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / per), c = (int)(i - (int64_t)r * per) * 4;
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = 0.f;
      if (c + q < cols) {
        const int64_t at = base + (int64_t)r * cols + c + q;
        const float m = M[at], u = nesterov ? fmaf(mu, m, Elt<T>::get(G + at)) : m;
        const double x = (double)u * inv;
        if constexpr (UPDATE) {
          const float y = fmaf(-us, (float)x, ws * Elt<T>::get(W + at));
          if constexpr (sizeof(T) == 4) {
            W[at] = y;
          } else {
            W[at] = f2bf(y);
          }
        } else {
          v[q] = (float)(x * (double)pow2(kXe));
        }
      }
    }
    if constexpr (!UPDATE) put4<LO>(o, mat * o.step + (int64_t)r * o.ld + c, 4, v);
  }
}

// ---- host ---------------------------------------------------------------------------
int32_t pad8(int32_t n) { return (n + 7) / 8 * 8; }

struct Bufs {
  double* part = nullptr;
  Planes x0{}, x1{}, a{}, b{};
  int parts = 0;
};

template <class Mem>
Planes planes(const hg_muon_desc* A, int32_t rows, int32_t cols, Mem& m) {
  Planes p{};
  p.rows = rows;
  p.cols = cols;
  p.ld = pad8(cols);
  p.step = (int64_t)rows * p.ld;
  p.lo = p.step * A->count;
  p.p = m.template take<uint16_t>(p.lo * (A->dtype == HG_DTYPE_F32 ? 2 : 1));
  return p;
}

template <class Mem>
Bufs take(const hg_muon_desc* A, Mem& m) {
  Bufs b;
  const int64_t n = (int64_t)A->rows * A->cols;
  const int32_t k = std::min(A->rows, A->cols);
  b.parts = (int)std::min<int64_t>(kNormBlocks, std::max<int64_t>(1, cdiv(n, 1024)));
  b.part = m.template take<double>((int64_t)A->count * b.parts);
  if (A->steps == 0) {
    b.x0.ld = pad8(A->cols);
    return b;
  }
  b.x0 = planes(A, A->rows, A->cols, m);
  if (A->steps > 1) b.x1 = planes(A, A->rows, A->cols, m);
  b.a = planes(A, k, k, m);
  b.b = planes(A, k, k, m);
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

template <bool AKM, bool BKM, int BM, int BN, int WM, int WN, bool LO, int EPI, class TW>
int product(const char* name, MuonArgs a, int count, hipStream_t s) {
  constexpr size_t bytes = 2 * (LO ? 2 : 1) * (size_t)(BM + BN) * 64 * 2;
  a.tiles_m = (a.M + BM - 1) / BM;
  a.tiles_n = (a.N + BN - 1) / BN;
  a.tiles = EPI <= kEpiSymAdd ? a.tiles_m * (a.tiles_m + 1) / 2 : a.tiles_m * a.tiles_n;
  constexpr auto kernel = k_muon_product<AKM, BKM, BM, BN, WM, WN, LO, EPI, TW>;
  HG_TRY(allow_lds<kernel>(bytes));
  HG_LAUNCH(name, kernel, dim3((unsigned)(a.tiles * count)), dim3((BM / WM) * (BN / WN) * 64), bytes, s, a);
  return HG_OK;
}

template <bool TALL, bool LO, class TW>
int steps(const hg_muon_desc* A, const Bufs& b, void* W, hipStream_t s) {
  Planes x = b.x0, next = b.x1;
  const int32_t k = std::min(A->rows, A->cols), len = std::max(A->rows, A->cols);
  for (int i = 0; i < A->steps; ++i) {
    MuonArgs g{};
    g.a = g.b = x;
    g.o = b.a;
    g.M = g.N = k;
    g.K = len;
    g.zs = pow2(kAe - 2 * kXe);
    HG_TRY((product<!TALL, !TALL, 64, 64, 32, 32, LO, kEpiSym, TW>("muon_gram", g, A->count, s)));
    g.a = g.b = g.c = b.a;
    g.o = b.b;
    g.K = k;
    g.zs = kS * pow2(kBe - 2 * kAe);
    g.cs = kQ * pow2(kBe - kAe);
    HG_TRY((product<true, true, 64, 64, 32, 32, LO, kEpiSymAdd, TW>("muon_square", g, A->count, s)));
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
      HG_TRY((product<true, TALL, 64, 64, 32, 32, LO, kEpiAdd, TW>("muon_apply", g, A->count, s)));
      std::swap(x, next);
    } else {
      g.W = W;
      g.ws = 1.f - A->lr * A->weight_decay;
      g.us = A->lr * A->scale * pow2(-kXe);
      HG_TRY((product<true, TALL, 64, 64, 32, 32, LO, kEpiUpdate, TW>("muon_update", g, A->count, s)));
    }
  }
  return HG_OK;
}

template <class T>
int run(const hg_muon_desc* A, const Bufs& b, T* W, const T* G, float* M, hipStream_t s) {
  constexpr bool LO = sizeof(T) == 4;
  const int64_t n = (int64_t)A->rows * A->cols;
  const dim3 grid((unsigned)b.parts, (unsigned)A->count);
  HG_LAUNCH("muon_momentum", k_muon_momentum<T>, grid, dim3(256), 0, s, G, M, n, A->mu, A->nesterov, b.part);
  if (A->steps == 0) {
    HG_LAUNCH("muon_first", (k_muon_first<T, LO, true>), grid, dim3(256), 0, s, G, M, A->rows, A->cols, A->mu, A->nesterov,
              b.part, b.parts, A->eps, b.x0, W, 1.f - A->lr * A->weight_decay, A->lr * A->scale);
    return HG_OK;
  }
  HG_LAUNCH("muon_first", (k_muon_first<T, LO, false>), grid, dim3(256), 0, s, G, M, A->rows, A->cols, A->mu, A->nesterov, b.part,
            b.parts, A->eps, b.x0, W, 0.f, 0.f);
  return A->rows > A->cols ? steps<true, LO, T>(A, b, W, s) : steps<false, LO, T>(A, b, W, s);
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
  const auto meet = [](const void* p, size_t a, const void* q, size_t b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
    return x < y + b && y < x + a;
  };
  if (meet(W, n * e, G, n * e) || meet(W, n * e, M, n * 4) || meet(G, n * e, M, n * 4))
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
