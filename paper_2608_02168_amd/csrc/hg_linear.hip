// Linear map with bias, activation and residual, and the gated product of a
// feed-forward block, forward and backward: operand preparation, the choice of
// tiles and the launches around the product core of hg_gemm.h.
//
//   linear   z = X W + b,       Y = act(z) + R
//   gated    [a u] = X W + b,   H = act(a) * u
//   backward dz from z and the upstream rows (the forward product once more,
//            with the gradient in its epilogue), dX = dz W^T, dW = X^T dz
//
// The gated product is the same product with the columns of a tile taken by
// 16 in turn from the gate and from the up projection, so that a lane holds
// both values of an output and z never leaves the registers.
//
// bfloat16 operands are used where they lie when their rows are 16-byte
// aligned and a multiple of 8 wide; else they are copied once into padded
// rows.  float32 operands are always used where they lie (split into parts on
// the way to LDS).

#include "hg_gemm.h"

namespace hg {
namespace {

// One call of either operator.
struct Prob {
  int64_t n;
  int32_t d, f;       // f: width of the output (of one half)
  int32_t dtype, act;
  bool gated;
  int64_t ld_x, ld_y, ld_r;
  int32_t halves() const { return gated ? 2 : 1; }
  int32_t cols() const { return halves() * f; }            // columns of W
  int32_t dp() const { return (d + 7) / 8 * 8; }
  int32_t fp() const { return f32() ? f : (f + 7) / 8 * 8; }  // width of a half in operands and in dz
  int32_t colsp() const { return halves() * fp(); }
  bool f32() const { return dtype == HG_DTYPE_F32; }
  int32_t parth() const { return (fp() + 3) / 4 * 4; }
  int64_t ld_part() const { return (int64_t)halves() * parth(); }
};

constexpr int32_t kMaxWidth = 1 << 20;
constexpr int64_t kMaxLd = 1 << 22;   // 256 rows of 16-bit values stay below 2^31 bytes

bool direct(int32_t width, int64_t ld) { return width % 8 == 0 && ld % 8 == 0 && ld < kMaxLd; }

// ---- preparation -----------------------------------------------------------------
// A padded row is `halves` halves of Fp values (a multiple of 8), each with F
// values of the source row side by side; the padding is zero.
struct RowShape {
  int32_t F, Fp, halves;
};

// bfloat16 rows into padded rows; a thread moves eight values.
__global__ void __launch_bounds__(256)
    k_rows_pad(const uint16_t* __restrict__ src, int64_t ld, int64_t rows, RowShape rs, uint16_t* __restrict__ dst) {
  const int chunks = rs.halves * rs.Fp / 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / chunks;
  if (row >= rows) return;
  const int j = (int)(id - row * chunks) * 8;
  const int h = j >= rs.Fp, f = j - h * rs.Fp;
  const uint16_t* p = src + row * ld + h * rs.F + f;
  uint16_t v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = f + q < rs.F ? p[q] : 0;
  uint4 o;
  __builtin_memcpy(&o, v, 16);
  *reinterpret_cast<uint4*>(dst + row * (int64_t)(rs.halves * rs.Fp) + j) = o;
}

// ---- column sums --------------------------------------------------------------------
constexpr int kSumRows = 256;  // rows that one block sums

template <class T>
__global__ void __launch_bounds__(256)
    k_colsum(const void* __restrict__ x, int64_t ld, int64_t rows, int32_t cols, float* __restrict__ part) {
  __shared__ float sh[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int col = blockIdx.y * 64 + lane;
  const int64_t r0 = (int64_t)blockIdx.x * kSumRows;
  const int64_t r1 = r0 + kSumRows < rows ? r0 + kSumRows : rows;
  float s = 0.f;
  if (col < cols)
    for (int64_t r = r0 + w; r < r1; r += 4) s += g_load1<T>(x, r * ld + col);
  sh[w][lane] = s;
  __syncthreads();
  if (w == 0 && col < cols) part[blockIdx.x * (int64_t)cols + col] = sh[0][lane] + sh[1][lane] + sh[2][lane] + sh[3][lane];
}

// Sums of `parts` rows of partial column sums: 16 columns a block, 64 threads a
// column (every 64th row in order, then the 64 sums in a fixed order).
__global__ void __launch_bounds__(1024)
    k_colsum_join(const float* __restrict__ part, int64_t parts, int32_t cols, float* __restrict__ out, int accumulate) {
  __shared__ float sh[16][17];
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + cx;
  float s = 0.f;
  if (col < cols)
#pragma unroll 8
    for (int64_t r = ry; r < parts; r += 64) s += part[r * cols + col];
  // four rows of the block lie in a wave
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if ((ry & 3) == 0) sh[ry >> 2][cx] = s;
  __syncthreads();
  if (ry == 0 && col < cols) {
#pragma unroll
    for (int q = 1; q < 16; ++q) s += sh[q][cx];
    out[col] = accumulate ? out[col] + s : s;
  }
}

// ---- few rows -------------------------------------------------------------------------
// Y of NR rows by reading W once: a lane takes 16 bytes of eight consecutive k
// rows (8 k x VEC columns) and the same eight k of every row of X, so a wave
// reads 8 x 64 rows' pieces, and the 8 waves of a block split k.  Bound by
// the bytes of W (33.5 MB in 11.8 us, 2.8 TB/s, where 4096 columns make 128
// blocks; 3.5 TB/s with 256).  LC lanes side by side cover LC * 16 bytes of a row.
constexpr int kFewWaves = 8;
constexpr int kFewRows = 8;  // at most

// 16 bytes of a row, n values of them inside.
template <class T, bool ALIGNED>
__device__ __forceinline__ typename Elt<T>::rawv_t few_load(const T* p, int n) {
  if (n >= Elt<T>::EL && ALIGNED) return Elt<T>::rawv(p);
  typename Elt<T>::rawv_t r = Elt<T>::rawv_zero();
  if constexpr (!ALIGNED) {
#pragma unroll
    for (int q = 0; q < Elt<T>::EL; ++q) {
      if (q >= n) continue;
      if constexpr (sizeof(T) == 4) {
        r[q] = p[q];
      } else {
        r[q >> 1] |= (uint32_t)p[q] << (16 * (q & 1));
      }
    }
  }
  return r;
}

template <class T, class Epi, int NR, int LC, bool ALIGNED>
__global__ void __launch_bounds__(kFewWaves * 64)
    k_few_rows(const T* __restrict__ X, int64_t ld_x, const T* __restrict__ W, int32_t K, int32_t f, int nr,
               const GEpi e) {
  constexpr int VEC = Elt<T>::EL, H = Epi::kGated ? 2 : 1, COLS = LC * VEC, KG = 64 / LC;
  __shared__ float sh[kFewWaves][H][NR][COLS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lc = lane % LC, kg = lane / LC;
  const int64_t ldw = (int64_t)H * f;
  // neighbouring column blocks to one XCD: they share the lines of W
  const uint32_t nb = gridDim.x, per = nb / 8, x = blockIdx.x % 8, more = nb % 8;
  const int c0 = (int)(x * per + (x < more ? x : more) + blockIdx.x / 8) * COLS;
  const int col = c0 + lc * VEC;
  const int cl = f - col;  // columns left
  float acc[H][NR][VEC];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int q = 0; q < VEC; ++q) acc[h][r][q] = 0.f;
  if (cl > 0) {
    for (int k = (wave * KG + kg) * 8; k < K; k += kFewWaves * KG * 8) {
      typename Elt<T>::rawv_t w[H][8], xv[NR][8 / VEC];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int h = 0; h < H; ++h)
          w[h][j] = few_load<T, ALIGNED>(W + (k + j < K ? k + j : k) * ldw + h * (int64_t)f + col, k + j < K ? cl : 0);
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int j = 0; j < 8; j += VEC)
          xv[r][j / VEC] = few_load<T, ALIGNED>(X + (r < nr ? r : 0) * ld_x + (k + j < K ? k + j : k), K - k - j);
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            const float xs = Elt<T>::rawv_get(xv[r][j / VEC], j % VEC);
#pragma unroll
            for (int q = 0; q < VEC; ++q) acc[h][r][q] = fmaf(xs, Elt<T>::rawv_get(w[h][j], q), acc[h][r][q]);
          }
    }
  }
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int q = 0; q < VEC; ++q) {
        float s = acc[h][r][q];
#pragma unroll
        for (int o = LC; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
        if (kg == 0) sh[wave][h][r][lc * VEC + q] = s;
      }
  __syncthreads();
  for (int t = threadIdx.x; t < NR * COLS / 4; t += kFewWaves * 64) {
    const int r = t / (COLS / 4), cc = t % (COLS / 4) * 4, n = c0 + cc;
    if (r >= nr || n >= f) continue;
    float z[H][4];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) s += sh[w][h][r][cc + q];
        z[h][q] = s;
      }
    float res[4];
    const GCols ec = Epi::cols(e, n);
    Epi::load(e, ec, r, res);
    g_by_act<Epi::kAct>(e.act, [&](auto act) {
      constexpr int ACT = decltype(act)::value;
      if constexpr (Epi::kGated) {
        Epi::template apply<ACT>(e, ec, r, z[0], z[H - 1], res);
      } else {
        Epi::template apply<ACT>(e, ec, r, z[0], res);
      }
    });
  }
}

template <class T, class Epi, int LC, bool ALIGNED>
int launch_few(const Prob& p, const T* X, const T* W, const GEpi& e, hipStream_t s) {
  const unsigned grid = (unsigned)cdiv(p.f, LC * Elt<T>::EL);
  const int nr = (int)p.n;
#define HG_FEW(NR_)                                                                                          \
  HG_LAUNCH("few_rows", (k_few_rows<T, Epi, NR_, LC, ALIGNED>), dim3(grid), dim3(kFewWaves * 64), 0, s, X,   \
            p.ld_x, W, p.d, p.f, nr, e)
  constexpr bool kBf = sizeof(T) == 2;
  if (nr == 1) {
    HG_FEW(1);
  } else if (nr == 2) {
    HG_FEW(2);
  } else if (!(kBf && ALIGNED) && nr <= 4) {
    if constexpr (!(kBf && ALIGNED)) HG_FEW(4);
  } else {
    if constexpr (kBf && !ALIGNED) HG_FEW(8);
  }
#undef HG_FEW
  return HG_OK;
}

// ---- tiles ----------------------------------------------------------------------------
struct Tiling {
  int tile;
  int64_t tiles_m, tiles_n;
  int splits;
  int64_t k_split;
};

// Tiles of 256 x 256 where they fill most of the chip, have at least 512 k for
// their long epilogue and count at most an eighth more padding than 128 x 128
// (SiLU, 40000 rows, 128 to 384 columns: backward 60 us, 91 without the last two
// conditions; 30000 rows, 256 to 1024: backward 123 us, 138 without the one on k,
// forward 41, 42; the gated forward of 256 to 2 x 512 loses by it, 34 us, 32).  Tiles of
// 128 x 128 where they fill half the chip and count less than half more padding than
// 64 x 64 (60000 rows, 304 to 64 columns: 11.3 us, 13.5 with tiles of 128; backward
// with SiLU 50, 58).  Up to `short_k` values of k a bfloat16 tile is mostly epilogue,
// and 64 x 64, of which twice as many waves fit a CU, are faster: 256 for the gradient
// of z, whose epilogue reads and writes (20000 rows, 160 to 520: backward 61 us, 73;
// gated, 200 to 600: 94, 101), 128 without that (40000 rows, 96 to 256: 12.1 us, 14.2),
// none for the gated product (30000 rows, 80 to 100: 13.6 us, 15.8 with 64).  The k
// range is split over blocks while the tiles do not fill the chip (never where
// column sums are formed on the way).
Tiling tiling(int64_t M, int64_t cols, int64_t K, bool may_split, bool f32, int64_t short_k) {
  Tiling t{};
  const auto tiles_of = [&](int64_t x) { return cdiv(M, x) * cdiv(cols, x); };
  const int64_t big = tiles_of(128), huge = tiles_of(256);
  if (!f32 && huge >= 192 && K >= 512 && 8 * 4 * huge <= 9 * big) {
    t = Tiling{256, cdiv(M, 256), cdiv(cols, 256), 1, cdiv(std::max<int64_t>(K, 1), 64) * 64};
    return t;
  }
  t.tile = (big >= 128 || (may_split && big * (K / 512) >= 128)) && 2 * 4 * big <= 3 * tiles_of(64) &&
                   (f32 || K > short_k)
               ? 128
               : 64;
  t.tiles_m = cdiv(M, t.tile);
  t.tiles_n = cdiv(cols, t.tile);
  const int64_t tiles = t.tiles_m * t.tiles_n;
  int64_t splits = 1;
  if (may_split && tiles < 256) splits = std::max<int64_t>(1, std::min(cdiv(512, tiles), K / 256));
  t.k_split = cdiv(cdiv(std::max<int64_t>(K, 1), splits), 64) * 64;
  t.splits = (int)std::max<int64_t>(1, cdiv(K, t.k_split));
  return t;
}

int64_t part_elems(const Tiling& t, int64_t M, int64_t ld, int planes = 1) {
  return t.splits * planes > 1 ? (int64_t)t.splits * planes * M * ld : 0;
}

template <bool AKM, bool BKM, int TILE, class Epi, bool SPLIT>
int launch_tiles(const char* name, const GArgs<uint16_t>& a, const Tiling& t, hipStream_t s) {
  constexpr size_t lds = g_lds_bytes(2, TILE, TILE, 64);
  constexpr int WN = TILE == 256 ? 64 : TILE / 2, NT = 2 * (TILE / WN) * 64;
  constexpr auto kern = k_gemm16<AKM, BKM, TILE, TILE, 64, TILE / 2, WN, Epi, SPLIT>;
  HG_TRY((allow_lds<kern, lds>()));
  HG_LAUNCH(name, kern, dim3((unsigned)(t.tiles_m * t.tiles_n), SPLIT ? t.splits : 1), dim3(NT), lds, s, a);
  return HG_OK;
}

template <bool AKM, bool BKM, int TILE, class Epi, bool SPLIT, bool VEC>
int launch_tiles32(const char* name, const GArgs<float>& a, const Tiling& t, hipStream_t s) {
  constexpr size_t lds = g_lds_bytes(3, TILE, TILE, kG32K);
  constexpr auto kern = k_gemm32<AKM, BKM, TILE, TILE, TILE / 2, TILE / 2, Epi, SPLIT, VEC>;
  HG_TRY((allow_lds<kern, lds>()));
  HG_LAUNCH(name, kern, dim3((unsigned)(t.tiles_m * t.tiles_n), SPLIT ? t.splits : 1), dim3(256), lds, s, a);
  return HG_OK;
}

// Whether every group of four values of a float32 operand is 16-byte aligned.
bool vec4(const GOperand<float>& o) {
  return (reinterpret_cast<uintptr_t>(o.p) & 15) == 0 && o.ld % 4 == 0 && o.cols % 4 == 0;
}

template <bool AKM, bool BKM, int TILE, class Epi, bool SPLIT>
int launch_tiles(const char* name, const GArgs<float>& a, const Tiling& t, hipStream_t s) {
  if (vec4(a.a) && vec4(a.b) && (!Epi::kGated || a.e.half % 4 == 0))
    return launch_tiles32<AKM, BKM, TILE, Epi, SPLIT, true>(name, a, t, s);
  return launch_tiles32<AKM, BKM, TILE, Epi, SPLIT, false>(name, a, t, s);
}

// The split launch only forms products: one kernel for every epilogue of a form.
template <bool GATED>
struct EpiPart {
  static constexpr bool kGated = GATED, kColSum = false, kAct = false;
};

// Whether an epilogue writes a gradient in two parts (tiles of 128 at most).
template <class Epi>
constexpr bool two_parts() {
  if constexpr (Epi::kColSum) return Epi::kLo;
  return false;
}

template <bool AKM, bool BKM, class Epi, class T>
int launch_product(const char* name, GArgs<T> a, const Tiling& t, float* part, int32_t parth, hipStream_t s) {
  a.tiles_m = (int32_t)t.tiles_m;
  a.tiles_n = (int32_t)t.tiles_n;
  a.k_split = t.k_split;
  Tiling u = t;  // the blocks of both planes
  if (a.lo_a || a.lo_b) {
    a.lo_from = (uint32_t)t.splits;
    u.splits = 2 * t.splits;
  }
  if (u.splits == 1) {
    if constexpr (sizeof(T) == 2 && !two_parts<Epi>())
      if (t.tile == 256) return launch_tiles<AKM, BKM, 256, Epi, false>(name, a, t, s);
    if (t.tile == 128) return launch_tiles<AKM, BKM, 128, Epi, false>(name, a, t, s);
    return launch_tiles<AKM, BKM, 64, Epi, false>(name, a, t, s);
  }
  if constexpr (!Epi::kColSum) {
    typedef EpiPart<Epi::kGated> Part;
    a.e.part = part;
    a.e.parth = parth;
    a.e.ld_part = (Epi::kGated ? 2 : 1) * (int64_t)parth;
    if (t.tile == 128) {
      HG_TRY((launch_tiles<AKM, BKM, 128, Part, true>(name, a, u, s)));
    } else {
      HG_TRY((launch_tiles<AKM, BKM, 64, Part, true>(name, a, u, s)));
    }
    const int64_t quads = a.M * cdiv(Epi::kGated ? a.e.halfp : a.N, 4);
    if (u.splits > 8) {
      HG_LAUNCH("product_join", (k_product_join<Epi, 8>), dim3((unsigned)cdiv(quads, 32)), dim3(256), 0, s, a, u.splits);
    } else {
      HG_LAUNCH("product_join", (k_product_join<Epi, 1>), dim3((unsigned)cdiv(quads, 256)), dim3(256), 0, s, a, u.splits);
    }
  }
  return HG_OK;
}

// ---- a call's buffers ---------------------------------------------------------------------
// The same takes size the workspace and hand it out.
struct Bufs {
  uint16_t* x16 = nullptr;  // X and W in padded rows (bfloat16 whose rows cannot be used where they lie)
  uint16_t* w16 = nullptr;
  void* dz = nullptr;       // gradient of z in dtype
  float* part = nullptr;    // split products
  float* colsum = nullptr;
  int64_t colsum_rows = 0;
};

// Few rows: up to 2 bfloat16 rows (4096 x 4096: 11.8 us for one, 13.5 by tiles with
// k split; 4 rows 16.3), 4 float32 rows (2048 x 2048: 8 rows 12.7 us, 9 by tiles
// 13.2), and 8 where W would have to be copied first.
bool few(const Prob& p) { return p.n <= (p.f32() ? 4 : p.f % 8 ? kFewRows : 2); }
Tiling t_fwd(const Prob& p) { return tiling(p.n, p.colsp(), p.d, true, p.f32(), p.gated ? 0 : 128); }
Tiling t_z(const Prob& p) { return tiling(p.n, p.colsp(), p.d, false, p.f32(), 256); }
Tiling t_dx(const Prob& p) { return tiling(p.n, p.d, p.colsp(), true, p.f32(), 128); }
Tiling t_dw(const Prob& p) { return tiling(p.d, p.colsp(), p.n, true, p.f32(), 0); }
bool x_direct(const Prob& p) { return p.f32() || direct(p.d, p.ld_x); }
bool w_direct(const Prob& p) { return p.f32() || p.f % 8 == 0; }
bool has_z(const Prob& p) { return p.gated || p.act != HG_ACT_NONE; }
// Parts (bfloat16 values) that a bfloat16 gradient of z is kept in.  One adds as much
// to the error of dX and dW as their own rounding (together 0.0023 of the norm,
// 0.0017 without; 0.0025 met among results of some hundred values, whose error
// varies most).  Two where a result has few values and the products are bound by
// their launches (10 rows, 24 to 1448: 33 us, 27 with one part; 60000 rows, 64 to
// 64, keep one: 30 us, 47 with two).  Never with tiles of 256.
int planes(const Prob& p) {
  return !p.f32() && has_z(p) && p.d * std::min<int64_t>(p.n, p.cols()) < 4096 &&
                 p.n * p.d <= ((int64_t)1 << 28) / p.cols()
             ? 2
             : 1;
}
// the upstream rows are dz itself and can be read where they lie
bool dz_direct(const Prob& p) { return !has_z(p) && (p.f32() || direct(p.f, p.ld_y)); }

// Narrow float32 rows whose backward is one pass: groups of four aligned, and
// several tiles for every block.  With SiLU in us, and by tiles:
//            16384 rows          200003 rows
//   128 -> 128    34 (48)            134 (202)
//    64 -> 64     22 (29)             75 (93)
//     4 -> 100    22 (34)             86 (107)
//    16 -> 16     21 (26)             67 (60)
// (the planes in LDS are 128 wide whatever the widths are: up to 32 wide very many rows
// lose a tenth, and 65536 are even).
bool narrow(const Prob& p) {
  return p.f32() && !p.gated && p.d <= kNarrow && p.f <= kNarrow && p.n >= 16384 && p.d % 4 == 0 && p.f % 4 == 0 &&
         p.ld_x % 4 == 0 && p.ld_y % 4 == 0 && p.ld_r % 4 == 0;
}
constexpr int kNarrowBlocks = 256;

template <class Mem>
void take_operands(const Prob& p, Mem& m, Bufs& b) {
  if (!x_direct(p)) b.x16 = m.template take<uint16_t>(p.n * p.dp());
  if (!w_direct(p)) b.w16 = m.template take<uint16_t>((int64_t)p.d * p.colsp());
}

template <class Mem>
Bufs take_fwd(const Prob& p, Mem& m) {
  Bufs b;
  if (p.n == 0 || few(p)) return b;
  take_operands(p, m, b);
  b.part = m.template take<float>(part_elems(t_fwd(p), p.n, p.ld_part()));
  return b;
}

int64_t pad4(int64_t x) { return (x + 3) / 4 * 4; }

template <class Mem>
Bufs take_bwd(const Prob& p, Mem& m) {
  Bufs b;
  if (p.n == 0) return b;
  take_operands(p, m, b);
  if (!dz_direct(p)) {
    if (p.f32()) {
      b.dz = m.template take<float>(p.n * p.colsp());
    } else {
      b.dz = m.template take<uint16_t>(planes(p) * p.n * p.colsp());
    }
  }
  b.colsum_rows = has_z(p) ? t_z(p).tiles_m : cdiv(p.n, kSumRows);
  // (a narrow call may still go by tiles: without dX, or to rows that are not aligned)
  const int64_t blocks = narrow(p) ? kNarrowBlocks : 0;
  b.colsum = m.template take<float>(std::max(b.colsum_rows, blocks) * p.cols());
  b.part = m.template take<float>(std::max({part_elems(t_dx(p), p.n, pad4(p.d), planes(p)),
                                            part_elems(t_dw(p), p.d, pad4(p.colsp()), planes(p)),
                                            blocks * p.d * p.f}));
  return b;
}

// ---- checks -----------------------------------------------------------------------------------
// A grid has fewer than 2^32 threads in x: of the tiles, and of the copies into padded
// rows, a thread for eight values.  (Joins and column sums have fewer: the k range is
// split only where there are few tiles.)
bool launchable(const Tiling& t) { return t.tiles_m * t.tiles_n * (t.tile == 256 ? 512 : 256) < (int64_t)1 << 32; }
bool launchable_pad(int64_t rows, int64_t width) { return rows * (width / 8) <= ((int64_t)1 << 32) - 256; }

bool launchable(const Prob& p, bool bwd) {
  if (p.n == 0 || (!bwd && few(p))) return true;
  if ((!x_direct(p) && !launchable_pad(p.n, p.dp())) || (!w_direct(p) && !launchable_pad(p.d, p.colsp()))) return false;
  if (!bwd) return launchable(t_fwd(p));
  if (!has_z(p) && !dz_direct(p) && !launchable_pad(p.n, p.colsp())) return false;
  return (!has_z(p) || launchable(t_z(p))) && launchable(t_dx(p)) && launchable(t_dw(p));
}

int check(const Prob& p, const char* what, bool bwd) {
  if (p.n < 0 || p.d < 1 || p.f < 1) return fail(HG_ERR_ARG, "%s: sizes n=%lld, %d -> %d", what, (long long)p.n, p.d, p.f);
  if (p.dtype != HG_DTYPE_F32 && p.dtype != HG_DTYPE_BF16) return fail(HG_ERR_ARG, "%s: dtype %d", what, p.dtype);
  if (p.act < HG_ACT_NONE || p.act > HG_ACT_GELU) return fail(HG_ERR_ARG, "%s: act %d", what, p.act);
  if (p.n >= (int64_t)1 << 31 || p.d > kMaxWidth || p.f > kMaxWidth)
    return fail(HG_ERR_UNSUPPORTED, "%s: n=%lld, %d -> %d is too large", what, (long long)p.n, p.d, p.f);
  if (!launchable(p, bwd))
    return fail(HG_ERR_UNSUPPORTED, "%s: n=%lld rows of %d -> %d are too many", what, (long long)p.n, p.d, p.f);
  return HG_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Whether [a, a + na) and [b, b + nb) share a byte.
bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  if (!a || !b) return false;
  const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
  return x < y + nb && y < x + na;
}

int64_t span(const Prob& p, int64_t rows, int64_t width, int64_t ld) {
  return rows > 0 ? ((rows - 1) * ld + width) * (p.f32() ? 4 : 2) : 0;
}

int check_rows(const Prob& p, const char* what, int64_t ld, int32_t width, const char* name) {
  if (p.n > 0 && (ld < width || ld > (int64_t)1 << 40))
    return fail(HG_ERR_ARG, "%s: rows of %s are %lld apart, %d wide", what, name, (long long)ld, width);
  return HG_OK;
}

// ---- launches -----------------------------------------------------------------------------------
int pad_rows(const void* src, int64_t ld, int64_t rows, RowShape rs, uint16_t* dst, hipStream_t s) {
  HG_LAUNCH("rows_pad", k_rows_pad, dim3((unsigned)cdiv(rows * (rs.halves * rs.Fp / 8), 256)), dim3(256), 0, s,
            static_cast<const uint16_t*>(src), ld, rows, rs, dst);
  return HG_OK;
}

RowShape x_shape(const Prob& p) { return RowShape{p.d, p.dp(), 1}; }
RowShape w_shape(const Prob& p) { return RowShape{p.f, p.fp(), p.halves()}; }

// X as rows of k, and W, which serves as k rows and as rows of k.
int operands(const Prob& p, const void* X, const void* W, const Bufs&, GOperand<float>& x, GOperand<float>& w, hipStream_t) {
  x = GOperand<float>{static_cast<const float*>(X), p.ld_x, p.n, p.d};
  w = GOperand<float>{static_cast<const float*>(W), p.cols(), p.d, p.cols()};
  return HG_OK;
}

int operands(const Prob& p, const void* X, const void* W, const Bufs& b, GOperand<bf16_t>& x, GOperand<bf16_t>& w,
             hipStream_t s) {
  x = GOperand<bf16_t>{static_cast<const bf16_t*>(X), p.ld_x, p.n, p.dp()};
  if (!x_direct(p)) {
    HG_TRY(pad_rows(X, p.ld_x, p.n, x_shape(p), b.x16, s));
    x.p = b.x16;
    x.ld = p.dp();
  }
  w = GOperand<bf16_t>{static_cast<const bf16_t*>(W), p.colsp(), p.d, p.colsp()};
  if (!w_direct(p)) {
    HG_TRY(pad_rows(W, p.cols(), p.d, w_shape(p), b.w16, s));
    w.p = b.w16;
  }
  return HG_OK;
}

GEpi epi_of(const Prob& p, const float* bias, const void* res, int64_t ld_res, void* out, int64_t ld_out) {
  GEpi e{};
  e.bias = bias;
  e.res = res;
  e.ld_res = ld_res;
  e.out = out;
  e.ld_out = ld_out;
  e.act = p.act;
  e.ncol = p.f;
  e.half = p.f;
  e.halfp = p.fp();
  e.outp = p.fp();
  return e;
}

template <class T, bool GATED>
int fwd_impl(const Prob& p, const void* X, const void* W, const float* bias, const void* R, void* Y, const Bufs& b,
             hipStream_t s) {
  typedef typename std::conditional<GATED, EpiGated<T>, EpiLinear<T>>::type Epi;
  GArgs<T> a{};
  a.e = epi_of(p, bias, R, p.ld_r, Y, p.ld_y);
  if (few(p)) {
    constexpr int LC = 4;
    constexpr int V = Elt<T>::EL;
    const bool al = p.f % V == 0 && p.d % V == 0 && p.ld_x % V == 0;
    const T *x = static_cast<const T*>(X), *w = static_cast<const T*>(W);
    return al ? launch_few<T, Epi, LC, true>(p, x, w, a.e, s) : launch_few<T, Epi, LC, false>(p, x, w, a.e, s);
  }
  HG_TRY(operands(p, X, W, b, a.a, a.b, s));
  a.M = p.n;
  a.N = p.colsp();
  a.K = a.a.cols;
  return launch_product<true, false, Epi>(GATED ? "glu" : "linear", a, t_fwd(p), b.part, p.parth(), s);
}

// The one pass of narrow rows, then the sums over its blocks.
int narrow_bwd(const Prob& p, const float* X, const float* W, const float* bias, const float* dY, float* dX, float* dW,
               float* dbias, int accumulate, const Bufs& b, hipStream_t s) {
  const GNarrow a{X,     W,       dY,  bias, dX,    p.ld_x, p.ld_y, p.ld_r, p.n, p.d, p.f,
                  p.act, b.part, dbias ? b.colsum : nullptr, p.f};
  if (p.d <= 64 && p.f <= 64) {
    HG_TRY((allow_lds<k_narrow_bwd<2>, kNarrowLds>()));
    HG_LAUNCH("linear_narrow_bwd", k_narrow_bwd<2>, dim3(kNarrowBlocks), dim3(kNarrowThreads), kNarrowLds, s, a);
  } else {
    HG_TRY((allow_lds<k_narrow_bwd<4>, kNarrowLds>()));
    HG_LAUNCH("linear_narrow_bwd", k_narrow_bwd<4>, dim3(kNarrowBlocks), dim3(kNarrowThreads), kNarrowLds, s, a);
  }
  GShape j{};
  j.M = p.d;
  j.N = p.f;
  j.e.out = dW;
  j.e.ld_out = j.e.ld_part = p.f;
  j.e.ncol = p.f;
  j.e.accumulate = accumulate;
  j.e.part = b.part;
  HG_LAUNCH("product_join", (k_product_join<EpiSum<float>, 8>), dim3((unsigned)cdiv((int64_t)p.d * p.f / 4, 32)), dim3(256), 0,
            s, j, kNarrowBlocks);
  if (dbias)
    HG_LAUNCH("colsum_join", k_colsum_join, dim3((unsigned)cdiv(p.f, 16)), dim3(1024), 0, s, b.colsum, (int64_t)kNarrowBlocks,
              p.f, dbias, accumulate);
  return HG_OK;
}

template <class T, bool GATED>
int bwd_impl(const Prob& p, const void* X, const void* W, const float* bias, const void* dY, void* dX, int64_t ld_dx,
             void* dW, float* dbias, int accumulate, const Bufs& b, hipStream_t s) {
  typedef typename std::conditional<GATED, EpiGatedGrad<T, false>, EpiLinearGrad<T, false>>::type EpiG;
  typedef typename std::conditional<GATED, EpiGatedGrad<T, true>, EpiLinearGrad<T, true>>::type EpiG2;
  if constexpr (sizeof(T) == 4 && !GATED) {
    if (narrow(p) && dX && dW && aligned16(dX))
      return narrow_bwd(p, static_cast<const float*>(X), static_cast<const float*>(W), bias, static_cast<const float*>(dY),
                        static_cast<float*>(dX), static_cast<float*>(dW), dbias, accumulate, b, s);
  }
  GOperand<T> x{}, w{};
  HG_TRY(operands(p, X, W, b, x, w, s));
  // dz, in rows of colsp (or where the upstream rows lie); its second part
  const int64_t lo = planes(p) == 2 ? p.n * p.colsp() : 0;
  GOperand<T> z{static_cast<const T*>(b.dz), p.colsp(), p.n, p.colsp()};
  if (has_z(p)) {
    GArgs<T> a{};
    a.a = x;
    a.b = w;
    a.M = p.n;
    a.N = p.colsp();
    a.K = x.cols;
    a.e = epi_of(p, bias, dY, p.ld_y, b.dz, p.colsp());
    a.e.colsum = dbias ? b.colsum : nullptr;
    a.e.ld_colsum = p.cols();
    a.e.lo = lo;
    const char* name = GATED ? "glu_dz" : "linear_dz";
    bool two = false;
    if constexpr (sizeof(T) == 2) {
      two = lo > 0;
      if (two) HG_TRY((launch_product<true, false, EpiG2>(name, a, t_z(p), nullptr, 0, s)));
    }
    if (!two) HG_TRY((launch_product<true, false, EpiG>(name, a, t_z(p), nullptr, 0, s)));
  } else {
    if (dbias)
      HG_LAUNCH("colsum", k_colsum<T>, dim3((unsigned)b.colsum_rows, (unsigned)cdiv(p.cols(), 64)), dim3(256), 0, s, dY,
                p.ld_y, p.n, p.cols(), b.colsum);
    if (dz_direct(p)) {
      z.p = static_cast<const T*>(dY);
      z.ld = p.ld_y;
    } else {
      HG_TRY(pad_rows(dY, p.ld_y, p.n, w_shape(p), static_cast<uint16_t*>(b.dz), s));
    }
  }
  if (dbias)
    HG_LAUNCH("colsum_join", k_colsum_join, dim3((unsigned)cdiv(p.cols(), 16)), dim3(1024), 0, s, b.colsum, b.colsum_rows,
              p.cols(), dbias, accumulate);
  if (dX) {
    GArgs<T> a{};
    a.a = z;
    a.b = w;
    a.M = p.n;
    a.N = p.d;
    a.K = p.colsp();
    a.e.out = dX;
    a.e.ld_out = ld_dx;
    a.e.ncol = p.d;
    a.lo_a = lo;
    HG_TRY((launch_product<true, true, EpiSum<T>>(GATED ? "glu_dx" : "linear_dx", a, t_dx(p), b.part, (int32_t)pad4(p.d), s)));
  }
  if (dW) {
    GArgs<T> a{};
    a.a = x;
    a.b = z;
    a.M = p.d;
    a.N = p.colsp();
    a.K = p.n;
    a.e.out = dW;
    a.e.ld_out = p.cols();
    a.e.ncol = p.cols();
    if (GATED && p.f != p.fp()) {
      a.e.half = p.f;
      a.e.halfp = p.fp();
    }
    a.e.accumulate = accumulate;
    a.lo_b = lo;
    HG_TRY((launch_product<false, false, EpiSum<T>>(GATED ? "glu_dw" : "linear_dw", a, t_dw(p), b.part,
                                                    (int32_t)pad4(p.colsp()), s)));
  }
  return HG_OK;
}

__global__ void __launch_bounds__(256) k_zero16(uint16_t* __restrict__ p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// Gradients of a call without rows: zero (added: nothing changes).
int empty_grads(const Prob& p, void* dW, float* dbias, int accumulate, hipStream_t s) {
  if (accumulate) return HG_OK;
  const int64_t n = (int64_t)p.d * p.cols();
  if (dW) {
    if (p.f32()) {
      HG_TRY(fill_f32(static_cast<float*>(dW), 0.f, n, s));
    } else {
      HG_LAUNCH("zero16", k_zero16, dim3((unsigned)std::min<int64_t>(2048, cdiv(n, 256))), dim3(256), 0, s,
                static_cast<uint16_t*>(dW), n);
    }
  }
  if (dbias) HG_TRY(fill_f32(dbias, 0.f, p.cols(), s));
  return HG_OK;
}

int forward(const Prob& p, const char* what, const void* X, const void* W, const float* bias, const void* R, void* Y,
            void* ws, size_t ws_bytes, hipStream_t s) {
  HG_TRY(check(p, what, false));
  HG_TRY(check_rows(p, what, p.ld_x, p.d, "X"));
  HG_TRY(check_rows(p, what, p.ld_y, p.f, "the output"));
  if (R) HG_TRY(check_rows(p, what, p.ld_r, p.f, "R"));
  if (p.n == 0) return HG_OK;
  if (!X || !W || !Y) return fail(HG_ERR_ARG, "%s: null pointer", what);
  if (!aligned16(X) || !aligned16(W)) return fail(HG_ERR_ARG, "%s: X and W must be 16-byte aligned", what);
  const int64_t ny = span(p, p.n, p.f, p.ld_y);
  if (overlap(Y, ny, X, span(p, p.n, p.d, p.ld_x)) || overlap(Y, ny, W, span(p, p.d, p.cols(), p.cols())) ||
      overlap(Y, ny, bias, 4 * (int64_t)p.cols()) ||
      (R != Y && overlap(Y, ny, R, span(p, p.n, p.f, p.ld_r))) || (R == Y && p.ld_r != p.ld_y))
    return fail(HG_ERR_ARG, "%s: the output overlaps an input", what);
  Sizer need;
  take_fwd(p, need);
  if (ws_bytes < need.used || (need.used && !ws))
    return fail(HG_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need.used);
  if (!aligned16(ws)) return fail(HG_ERR_ARG, "%s: the workspace is not 16-byte aligned", what);
  Arena m(ws, ws_bytes);
  const Bufs b = take_fwd(p, m);
  if (p.f32())
    return p.gated ? fwd_impl<float, true>(p, X, W, bias, R, Y, b, s)
                   : fwd_impl<float, false>(p, X, W, bias, R, Y, b, s);
  return p.gated ? fwd_impl<bf16_t, true>(p, X, W, bias, R, Y, b, s)
                 : fwd_impl<bf16_t, false>(p, X, W, bias, R, Y, b, s);
}

int backward(const Prob& p, const char* what, const void* X, const void* W, const float* bias, const void* dY, void* dX,
             void* dW, float* dbias, int accumulate, void* ws, size_t ws_bytes, hipStream_t s) {
  HG_TRY(check(p, what, true));
  if (accumulate != 0 && accumulate != 1) return fail(HG_ERR_ARG, "%s: accumulate %d", what, accumulate);
  HG_TRY(check_rows(p, what, p.ld_x, p.d, "X"));
  HG_TRY(check_rows(p, what, p.ld_y, p.f, "the upstream gradient"));
  if (dX) HG_TRY(check_rows(p, what, p.ld_r, p.d, "dX"));
  if (p.n == 0) return empty_grads(p, dW, dbias, accumulate, s);
  if (!X || !W || !dY) return fail(HG_ERR_ARG, "%s: null pointer", what);
  if (!aligned16(X) || !aligned16(W) || !aligned16(dY))
    return fail(HG_ERR_ARG, "%s: X, W and the upstream gradient must be 16-byte aligned", what);
  const int64_t nx = span(p, p.n, p.d, p.ld_x), nw = span(p, p.d, p.cols(), p.cols()), ny = span(p, p.n, p.f, p.ld_y);
  const int64_t ndx = span(p, p.n, p.d, p.ld_r), nb = 4 * (int64_t)p.cols();
  const struct {
    const void* p;
    int64_t n;
  } out[3] = {{dX, ndx}, {dW, nw}, {dbias, nb}};
  for (int i = 0; i < 3; ++i) {
    if (overlap(out[i].p, out[i].n, X, nx) || overlap(out[i].p, out[i].n, W, nw) || overlap(out[i].p, out[i].n, dY, ny) ||
        overlap(out[i].p, out[i].n, bias, nb))
      return fail(HG_ERR_ARG, "%s: a gradient overlaps an input", what);
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return fail(HG_ERR_ARG, "%s: two gradients overlap", what);
  }
  Sizer need;
  take_bwd(p, need);
  if (ws_bytes < need.used || (need.used && !ws))
    return fail(HG_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need.used);
  if (!aligned16(ws)) return fail(HG_ERR_ARG, "%s: the workspace is not 16-byte aligned", what);
  Arena m(ws, ws_bytes);
  const Bufs b = take_bwd(p, m);
  if (p.f32())
    return p.gated ? bwd_impl<float, true>(p, X, W, bias, dY, dX, p.ld_r, dW, dbias, accumulate, b, s)
                   : bwd_impl<float, false>(p, X, W, bias, dY, dX, p.ld_r, dW, dbias, accumulate, b, s);
  return p.gated ? bwd_impl<bf16_t, true>(p, X, W, bias, dY, dX, p.ld_r, dW, dbias, accumulate, b, s)
                 : bwd_impl<bf16_t, false>(p, X, W, bias, dY, dX, p.ld_r, dW, dbias, accumulate, b, s);
}

Prob prob_of(const hg_linear_desc* L) {
  return Prob{L->n, L->d_in, L->d_out, L->dtype, L->act, false, L->ld_x, L->ld_y, L->ld_r};
}
Prob prob_of(const hg_glu_desc* L) { return Prob{L->n, L->d, L->f, L->dtype, L->act, true, L->ld_x, L->ld_h, L->ld_dx}; }

template <class D>
size_t size_of(const D* L, bool bwd) {
  if (!L) return 0;
  const Prob p = prob_of(L);
  if (check(p, "workspace size", bwd) != HG_OK) return 0;
  Sizer m;
  if (bwd) {
    take_bwd(p, m);
  } else {
    take_fwd(p, m);
  }
  return m.used;
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" size_t hg_linear_fwd_workspace_size(const hg_linear_desc* L) { return size_of(L, false); }
extern "C" size_t hg_linear_bwd_workspace_size(const hg_linear_desc* L) { return size_of(L, true); }
extern "C" size_t hg_glu_fwd_workspace_size(const hg_glu_desc* L) { return size_of(L, false); }
extern "C" size_t hg_glu_bwd_workspace_size(const hg_glu_desc* L) { return size_of(L, true); }

extern "C" int hg_linear_fwd(const hg_linear_desc* L, const void* X, const void* W, const float* bias, const void* R,
                             void* Y, void* ws, size_t ws_bytes, void* stream) {
  if (!L) return fail(HG_ERR_ARG, "hg_linear_fwd: null descriptor");
  return forward(prob_of(L), "hg_linear_fwd", X, W, bias, R, Y, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int hg_linear_bwd(const hg_linear_desc* L, const void* X, const void* W, const float* bias, const void* dY,
                             void* dX, void* dW, float* dbias, int32_t accumulate, void* ws, size_t ws_bytes,
                             void* stream) {
  if (!L) return fail(HG_ERR_ARG, "hg_linear_bwd: null descriptor");
  return backward(prob_of(L), "hg_linear_bwd", X, W, bias, dY, dX, dW, dbias, accumulate, ws, ws_bytes,
                  static_cast<hipStream_t>(stream));
}

extern "C" int hg_glu_fwd(const hg_glu_desc* L, const void* X, const void* W, const float* bias, void* H, void* ws,
                          size_t ws_bytes, void* stream) {
  if (!L) return fail(HG_ERR_ARG, "hg_glu_fwd: null descriptor");
  return forward(prob_of(L), "hg_glu_fwd", X, W, bias, nullptr, H, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int hg_glu_bwd(const hg_glu_desc* L, const void* X, const void* W, const float* bias, const void* dH, void* dX,
                          void* dW, float* dbias, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  if (!L) return fail(HG_ERR_ARG, "hg_glu_bwd: null descriptor");
  return backward(prob_of(L), "hg_glu_bwd", X, W, bias, dH, dX, dW, dbias, accumulate, ws, ws_bytes,
                  static_cast<hipStream_t>(stream));
}
