// Tiled matrix product on the bfloat16 MFMA with a fused epilogue: the core of
// the linear map and of the gated product, forward and backward.
//
//   Z[m][n] = sum_k A[m][k] B[k][n]
//
// Each operand is read as it lies: k contiguous (KM, "rows of k") or k the row index (the rows run over
// m or n).  That gives the three products of a linear map without a
// transposition pass:
//   z  = x W      A = x   KM,      B = W   k-rows
//   dx = dz W^T   A = dz  KM,      B = W   KM
//   dW = x^T dz   A = x   k-rows,  B = dz  k-rows
//
// A block of waves owns a BM x BN tile of Z and walks k in steps of BK with
// two LDS buffers: the tile of step t+1 is written to LDS by the loads
// themselves (buffer_load ... lds, 16 bytes a lane) while the MFMAs of step t
// run, one barrier a step.  Buffer descriptors carry the bounds: what lies
// past the last row reads as zero.
//
// LDS layouts (a load writes 64 x 16 consecutive bytes, so a swizzle has to be
// in the global address of the lane):
//   KM      [row][BK]: the 16-byte chunk ch of row r lies at slot ch ^ (r & 7),
//           so the 16 rows that one fragment read touches fall on all banks;
//   k-rows  [k][BM]: the 32-byte granule gr of row k lies at granule
//           gr ^ g_swz(k), for the transposing 8-byte reads, whose half wave
//           touches rows 0-3 and 8-11 of one granule.
//
// Bound by the MFMA where k is long: the backward of the gated product of 8192
// rows, 2048 to 2 x 8192, runs its three products at 1.10 PFLOP/s (1500 us); large
// products of the library reach 1.24 to 1.35 on this card.  With less than some
// hundred k the epilogue's rows bound it.
//
// The fragments enter the MFMA as (B, A), so lane (c, g) of the wave holds
// Z[16 i + c][16 j + 4 g + v], v = 0..3: four consecutive columns of a row.
#pragma once

#include "hg_mfma.h"

namespace hg {

typedef short g_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 g_bf16x4 __attribute__((ext_vector_type(4)));

// One operand.  KM: `rows` rows (m or n) of K values; else K rows of `cols`
// values.  ld in elements.  bfloat16: p 16-byte aligned, ld, K (KM) or cols
// multiples of 8.
template <class T>
struct GOperand {
  const T* p;
  int64_t ld;
  int64_t rows;  // rows of the matrix as stored
  int32_t cols;  // valid values of a row
};

// How Z becomes the output.
struct GEpi {
  const float* bias;  // [N] (gated: [2 F]) or null
  const void* res;    // residual rows (linear) or upstream gradient rows (backward), or null
  int64_t ld_res;
  void* out;
  int64_t ld_out;
  int32_t act;
  int32_t ncol;       // columns that the output has (the tiles may count padding too)
  int32_t half;       // gated: F; a [., 2 F] result stored in two padded halves: F; else 0
  int32_t halfp;      // distance of the two halves as the operands hold them
  int32_t outp;       // gradient of z: width of a row (gated: of each half) with its padding
  int32_t accumulate;
  float* colsum;      // [tiles of m][ld_colsum] column sums of what a tile wrote, or null
  int64_t ld_colsum;
  float* part;        // [splits][M][ld_part] when the k range is split
  int64_t ld_part;    // a multiple of 4
  int32_t parth;      // distance of the two halves in it, a multiple of 4
  int64_t lo;         // gradient of z in two bfloat16 parts: values from out to the second
};

struct GShape {
  int64_t M;
  int32_t N;          // columns of Z as the tiles count them (gated: 2 * halfp)
  int64_t K;
  int64_t k_split;    // k range of a split (a multiple of 64), >= K: no split
  int32_t tiles_m, tiles_n;
  GEpi e;
};
template <class T>
struct GArgs : GShape {
  GOperand<T> a, b;
  // split bfloat16 products whose A or B is the sum of two planes: values from the
  // first to the second, and the split from which on the second is taken (0: one plane)
  int64_t lo_a, lo_b;
  uint32_t lo_from;
};

// exp: 2^h of the rounded h = x log2 e from the hardware, corrected by the factor
// 1 + l ln 2 for what the rounding left (as a factor, since 2^h is infinite from
// x = 88.72 on, and adding l ln 2 times it would be NaN); relative error below 2^-22.
__device__ __forceinline__ float g_exp(float x) {
  constexpr float kLog2e = 1.4426950408889634f;
  x = __builtin_amdgcn_fmed3f(x, -150.f, 150.f);  // (so that l is a number)
  const float h = x * kLog2e, l = fmaf(x, 1.9259629911e-8f, fmaf(x, kLog2e, -h));
  return __builtin_amdgcn_exp2f(h) * fmaf(l, 0.69314718056f, 1.f);
}

__device__ __forceinline__ float g_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + g_exp(-z)); }

// Phi(z) = (1 + erf(z / sqrt 2)) / 2 with e = exp(-z^2 / 2).  The tail Phi(-x) is e
// times a polynomial in t = 1 / (1 + 0.3053 x), fitted to the least relative error
// over x = 0 .. 14.5 (7e-8; 2^-21 with its roundings): z Phi(z) keeps its digits for
// negative z, where 1 + erf cancels.
__device__ __forceinline__ float g_phi(float z, float e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.30525768f, fabsf(z), 1.f));
  float q = fmaf(t, 0.036317758f, -0.15108745f);
  q = fmaf(t, q, 0.18200397f);
  q = fmaf(t, q, -0.034953609f);
  q = fmaf(t, q, 0.11956811f);
  q = fmaf(t, q, 0.10389225f);
  q = fmaf(t, q, 0.12251315f);
  q = fmaf(t, q, 0.12174579f);
  const float tail = t * q * e;
  return z < 0.f ? tail : 1.f - tail;
}

// act of four values and, with G, its slopes
template <int ACT, bool G>
__device__ __forceinline__ void g_act4(const float (&z)[4], float (&f)[4], float (&d)[4]) {
  if constexpr (ACT == HG_ACT_SILU) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float s = g_sigmoid(z[q]);
      f[q] = z[q] * s;
      if (G) d[q] = fmaf(f[q], 1.f - s, s);
    }
  } else if constexpr (ACT == HG_ACT_GELU) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float e = g_exp(-0.5f * z[q] * z[q]), p = g_phi(z[q], e);
      f[q] = z[q] * p;
      if (G) d[q] = fmaf(z[q] * e, 0.39894228040143268f, p);
    }
  } else if constexpr (ACT == HG_ACT_RELU) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool nan = z[q] != z[q];
      f[q] = z[q] > 0.f || nan ? z[q] : 0.f;
      if (G) d[q] = nan ? z[q] : z[q] > 0.f ? 1.f : 0.f;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f[q] = z[q];
      if (G) d[q] = 1.f;
    }
  }
}

template <class T>
__device__ __forceinline__ float g_load1(const void* p, int64_t at) {
  if constexpr (sizeof(T) == 4) {
    return static_cast<const float*>(p)[at];
  } else {
    return bf2f(static_cast<const uint16_t*>(p)[at]);
  }
}

// Four consecutive values of a row; `vec`: they are all inside and aligned.
template <class T>
__device__ __forceinline__ void g_load4(const void* p, int64_t at, int n, bool vec, float (&v)[4]) {
  if (vec) {
    const f32x4 x = Elt<T>::load4(static_cast<const T*>(p) + at);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = x[q];
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = q < n ? g_load1<T>(p, at + q) : 0.f;
  }
}

template <class T>
__device__ __forceinline__ void g_store4(void* p, int64_t at, int n, bool vec, const float (&v)[4]) {
  if constexpr (sizeof(T) == 4) {
    float* o = static_cast<float*>(p) + at;
    if (vec) {
      *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < n) o[q] = v[q];
    }
  } else {
    uint16_t* o = static_cast<uint16_t*>(p) + at;
    if (vec) {
      *reinterpret_cast<uint2*>(o) = __builtin_bit_cast(uint2, __builtin_convertvector((f32x4{v[0], v[1], v[2], v[3]}), g_bf16x4));
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < n) o[q] = f2bf(v[q]);
    }
  }
}

// What bfloat16 rounding took from the values, into the second plane.
template <class T>
__device__ __forceinline__ void g_store_lo(const GEpi& e, int64_t at, int n, bool vec, const float (&v)[4]) {
  float l[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) l[q] = v[q] - bf2f(f2bf(v[q]));
  g_store4<T>(e.out, at + e.lo, n, vec, l);
}

// Rows whose four-value groups can be moved at once.
template <class T>
__device__ __forceinline__ bool g_vec(const void* p, int64_t ld) {
  return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (int64_t)sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
}

// Calls f with the launch's activation as a constant: a branch once, so that the
// code of one activation is in a row.
template <bool ACT, class F>
__device__ __forceinline__ void g_by_act(int act, F f) {
  if constexpr (!ACT) {
    f(std::integral_constant<int, HG_ACT_NONE>{});
  } else {
    switch (act) {
      case HG_ACT_RELU: f(std::integral_constant<int, HG_ACT_RELU>{}); break;
      case HG_ACT_SILU: f(std::integral_constant<int, HG_ACT_SILU>{}); break;
      case HG_ACT_GELU: f(std::integral_constant<int, HG_ACT_GELU>{}); break;
      default: f(std::integral_constant<int, HG_ACT_NONE>{});
    }
  }
}

// ---- epilogues: rows m, columns n .. n + 3 of Z --------------------------------
// `cols` is made once for a thread's columns; `load` reads what a row's output
// needs beside z; `apply` writes the output and replaces z by what it wrote (for
// the column sums).
struct GCols {
  int n, left;       // first column, columns from there on that exist
  int out;           // column of the output
  bool vr, vo, vo2;  // groups of four of res and of the output (of both halves) can be moved at once
  float b[4], b2[4];
};

template <class T>
__device__ __forceinline__ GCols g_cols(const GEpi& e, int n, int left, bool gated) {
  GCols c;
  c.n = c.out = n;
  c.left = left;
  c.vr = left >= 4 && g_vec<T>(e.res, e.ld_res);
  c.vo = left >= 4 && g_vec<T>(e.out, e.ld_out);
  c.vo2 = false;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    c.b[q] = e.bias && q < left ? e.bias[n + q] : 0.f;
    c.b2[q] = gated && e.bias && q < left ? e.bias[e.half + n + q] : 0.f;
  }
  return c;
}

template <class T>
__device__ __forceinline__ void g_load_res(const GEpi& e, const GCols& c, int64_t m, float (&r)[4]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) r[q] = 0.f;
  if (e.res) g_load4<T>(e.res, m * e.ld_res + c.n, c.left, c.vr, r);
}

// out = act(z + bias) + res
template <class T>
struct EpiLinear {
  static constexpr bool kGated = false, kColSum = false, kAct = true;
  __device__ static __forceinline__ GCols cols(const GEpi& e, int n) { return g_cols<T>(e, n, e.ncol - n, false); }
  __device__ static __forceinline__ void load(const GEpi& e, const GCols& c, int64_t m, float (&r)[4]) {
    g_load_res<T>(e, c, m, r);
  }
  template <int ACT>
  __device__ static __forceinline__ void apply(const GEpi& e, const GCols& c, int64_t m, float (&z)[4], const float (&r)[4]) {
    float f[4], d[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) z[q] += c.b[q];
    g_act4<ACT, false>(z, f, d);
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] += r[q];
    g_store4<T>(e.out, m * e.ld_out + c.n, c.left, c.vo, f);
  }
};

// out = res * act'(z + bias): the gradient of z; the padding of a row is written as zero
template <class T, bool LO>
struct EpiLinearGrad {
  static constexpr bool kLo = LO;  // in two parts
  static constexpr bool kGated = false, kColSum = true, kAct = true;
  __device__ static __forceinline__ GCols cols(const GEpi& e, int n) {
    GCols c = g_cols<T>(e, n, e.ncol - n, false);
    c.vo = e.outp - n >= 4 && g_vec<T>(e.out, e.ld_out);
    return c;
  }
  __device__ static __forceinline__ void load(const GEpi& e, const GCols& c, int64_t m, float (&r)[4]) {
    g_load_res<T>(e, c, m, r);
  }
  template <int ACT>
  __device__ static __forceinline__ void apply(const GEpi& e, const GCols& c, int64_t m, float (&z)[4], const float (&r)[4]) {
    float f[4], d[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) z[q] += c.b[q];
    g_act4<ACT, true>(z, f, d);
#pragma unroll
    for (int q = 0; q < 4; ++q) z[q] = q < c.left ? r[q] * d[q] : 0.f;
    g_store4<T>(e.out, m * e.ld_out + c.n, e.outp - c.n, c.vo, z);
    if constexpr (LO) g_store_lo<T>(e, m * e.ld_out + c.n, e.outp - c.n, c.vo, z);
  }
};

// out = z, or out + z; with half: the columns of two padded halves to [., 2 half]
template <class T>
struct EpiSum {
  static constexpr bool kGated = false, kColSum = false, kAct = false;
  __device__ static __forceinline__ GCols cols(const GEpi& e, int n) {
    GCols c;
    c.n = c.out = n;
    c.left = e.ncol - n;
    if (e.half) {
      // halfp is a multiple of 8, so four columns lie in one half
      const bool up = n >= e.halfp;
      c.left = e.half - (n - (up ? e.halfp : 0));
      c.out = n + (up ? e.half - e.halfp : 0);
    }
    c.vo = c.left >= 4 && g_vec<T>(e.out, e.ld_out) && (c.out & 3) == 0;
    return c;
  }
  __device__ static __forceinline__ void load(const GEpi& e, const GCols& c, int64_t m, float (&r)[4]) {
    if (e.accumulate) g_load4<T>(e.out, m * e.ld_out + c.out, c.left, c.vo, r);
  }
  template <int ACT>
  __device__ static __forceinline__ void apply(const GEpi& e, const GCols& c, int64_t m, float (&z)[4], const float (&r)[4]) {
    if (c.left <= 0) return;
    if (e.accumulate) {
#pragma unroll
      for (int q = 0; q < 4; ++q) z[q] += r[q];
    }
    g_store4<T>(e.out, m * e.ld_out + c.out, c.left, c.vo, z);
  }
};

// out = act(a + bias) * (u + bias), a and u the two halves' products
template <class T>
struct EpiGated {
  static constexpr bool kGated = true, kColSum = false, kAct = true;
  __device__ static __forceinline__ GCols cols(const GEpi& e, int n) { return g_cols<T>(e, n, e.half - n, true); }
  __device__ static __forceinline__ void load(const GEpi&, const GCols&, int64_t, float (&)[4]) {}
  template <int ACT>
  __device__ static __forceinline__ void apply(const GEpi& e, const GCols& c, int64_t m, float (&a)[4], float (&u)[4],
                                               const float (&)[4]) {
    if (c.left <= 0) return;
    float f[4], d[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) a[q] += c.b[q];
    g_act4<ACT, false>(a, f, d);
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] *= u[q] + c.b2[q];
    g_store4<T>(e.out, m * e.ld_out + c.n, c.left, c.vo, f);
  }
};

// da = dh u act'(a), du = dh act(a), side by side; the padding of a half is written as zero
template <class T, bool LO>
struct EpiGatedGrad {
  static constexpr bool kLo = LO;  // in two parts
  static constexpr bool kGated = true, kColSum = true, kAct = true;
  __device__ static __forceinline__ GCols cols(const GEpi& e, int n) {
    GCols c = g_cols<T>(e, n, e.half - n, true);
    c.vo = e.outp - n >= 4 && g_vec<T>(e.out, e.ld_out) && (e.outp & 3) == 0;
    return c;
  }
  __device__ static __forceinline__ void load(const GEpi& e, const GCols& c, int64_t m, float (&r)[4]) {
    g_load_res<T>(e, c, m, r);
  }
  template <int ACT>
  __device__ static __forceinline__ void apply(const GEpi& e, const GCols& c, int64_t m, float (&a)[4], float (&u)[4],
                                               const float (&r)[4]) {
    float f[4], d[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) a[q] += c.b[q];
    g_act4<ACT, true>(a, f, d);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool in = q < c.left;
      a[q] = in ? r[q] * (u[q] + c.b2[q]) * d[q] : 0.f;
      u[q] = in ? r[q] * f[q] : 0.f;
    }
    const int64_t at = m * e.ld_out + c.n;
    g_store4<T>(e.out, at, e.outp - c.n, c.vo, a);
    g_store4<T>(e.out, at + e.outp, e.outp - c.n, c.vo, u);
    if constexpr (LO) g_store_lo<T>(e, at, e.outp - c.n, c.vo, a);
    if constexpr (LO) g_store_lo<T>(e, at + e.outp, e.outp - c.n, c.vo, u);
  }
};

// ---- tile loads ----------------------------------------------------------------
// Raw buffer descriptor: an offset at or past `bytes` reads as zero.
__device__ __forceinline__ u32x4 g_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xFFFF),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}

// 16 bytes a lane from base + voff to LDS address lds + 16 * lane.  Written as
// an instruction, since the compiler would let every later LDS read wait for
// it: the caller waits (g_wait_loads) before the barrier that hands the buffer
// over.  It has no result register.  The compiler does not look into the block
// for what has to lie apart, so the block keeps it apart itself: one wait state
// from the write of m0 to the load that takes its LDS address from it, five from
// a vector instruction's write of a scalar register to a load that reads it (the
// descriptor's words may come from v_readfirstlane).
__device__ __forceinline__ void g_load_lds(u32x4 rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc)
               : "memory");
}
__device__ __forceinline__ void g_wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ uint32_t g_lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// The granule swizzle of k-row tiles: rows of 256 bytes and more, or of 128
// (four granules; the parity of the row is then half of the bank already).
template <int BM>
__device__ __forceinline__ int g_swz(int k) {
  if constexpr (BM >= 128) {
    return (k & 3) | (((k >> 3) & 1) << 2);
  } else {
    return ((k >> 1) & 1) | (((k >> 3) & 1) << 1);
  }
}

// One operand's share of a step, per wave: PER loads of 1 KB.
template <int BM, int BK, bool KM, int NW, bool GATED>
struct GTile {
  static constexpr int kBytes = BM * BK * 2;
  static constexpr int INSTR = kBytes / 1024, PER = INSTR / NW;
  static_assert(INSTR % NW == 0, "whole loads per wave");
  static_assert(!KM || BK == 64, "the chunk swizzle is made for 128-byte rows");
  uint32_t voff[PER];  // byte offset of the lane's 16 bytes from the step's base
  int kch;             // KM: first k of the lane's chunk (the same in every load)

  __device__ __forceinline__ void init(const GOperand<uint16_t>& o, int wave, int lane, int upper) {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int u = wave * PER + q;
      if constexpr (KM) {
        const int row = 8 * u + (lane >> 3), ch = (lane & 7) ^ (lane >> 3);
        voff[q] = (uint32_t)((row * o.ld + ch * 8) * 2);
        kch = ch * 8;
      } else {
        constexpr int SL = BM / 8, RPI = 64 / SL;  // 16-byte slots of a row, rows of a load
        const int row = RPI * u + lane / SL, slot = lane % SL;
        const int gr = (slot >> 1) ^ g_swz<BM>(row);
        const int col = GATED ? (gr >> 1) * 16 + (gr & 1) * upper : gr * 16;
        voff[q] = (uint32_t)((row * o.ld + col + (slot & 1) * 8) * 2);
        kch = 0;
      }
    }
  }
  // base: address of (row0, k0) or (k0, col0); left: bytes from there to the end of the last row
  __device__ __forceinline__ void issue(const uint16_t* base, int64_t left, int64_t k_left, uint32_t lds, int wave) const {
    const int64_t most = 0x7FFFFFF0;
    const u32x4 rsrc = g_rsrc(base, (uint32_t)(left < 0 ? 0 : (left < most ? left : most)));
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const uint32_t v = (KM && kch >= k_left) ? 0x7FFFFFF8u : voff[q];
      g_load_lds(rsrc, v, lds + (wave * PER + q) * 1024);
    }
  }
  // fragment of rows 16 i + c, k = 32 kb + 8 g .. + 7
  __device__ static __forceinline__ uint4 frag(const char* lds, int i, int kb, int c, int g) {
    if constexpr (KM) {
      const int row = 16 * i + c, ch = (4 * kb + g) ^ (c & 7);
      return *reinterpret_cast<const uint4*>(lds + row * 128 + ch * 16);
    } else {
      typedef __attribute__((address_space(3))) g_s16x4* lds_ptr;
      const int f = g_swz<BM>(8 * g + (c >> 2));
      const char* q = lds + (32 * kb + 8 * g + (c >> 2)) * (BM * 2) + ((i ^ f) * 32) + (c & 3) * 8;
      const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(q)));
      const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(q + 4 * BM * 2)));
      return uint4{a.x, a.y, b.x, b.y};
    }
  }
};

// XCD-aware order of the tiles: blocks go to the eight XCDs in turn, so each
// XCD takes one contiguous share of a walk that goes down `group` tile rows
// before it moves to the next tile column (operand tiles meet in its L2).
__device__ __forceinline__ void g_tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t group, uint32_t& im,
                                          uint32_t& in) {
  const uint32_t n = tm * tn, per = n / 8, more = n % 8;
  const uint32_t x = id % 8, at = id / 8;
  const uint32_t i = x * per + (x < more ? x : more) + at;
  const uint32_t span = group * tn, b = i / span, first = b * group;
  const uint32_t rows = tm - first < group ? tm - first : group;
  const uint32_t j = i - b * span;
  im = first + j % rows;
  in = j / rows;
}

// Rows of a tile that the epilogue holds in LDS at a time, and the LDS of a block.
constexpr int g_slab_rows(int bm, int bn) { return bm * (bn + 4) * 4 <= 70000 ? bm : 64; }
constexpr size_t g_lds_bytes(int stages, int bm, int bn, int bk) {
  const size_t a = (size_t)stages * (bm + bn) * bk * 2, b = (size_t)g_slab_rows(bm, bn) * (bn + 4) * 4;
  return a > b ? a : b;
}

// The tile of Z in the waves' accumulators to the output.  zt: the block's LDS.
template <int BM, int BN, int WM, int WN, class Epi, bool SPLIT>
__device__ __forceinline__ void g_epilogue(const GShape& p, const f32x4 (&acc)[WM / 16][WN / 16], float* zt, uint32_t im,
                                           int64_t m0, int n0, int bcol, int wm, int wn, int c, int g) {
  constexpr bool GATED = Epi::kGated;
  constexpr int MI = WM / 16, NI = WN / 16, NW = (BM / WM) * (BN / WN);
  // ---- epilogue: the tile goes through LDS in slabs of SR rows, so that rows
  // are read and written whole; a thread keeps its four columns of Z
  constexpr int SR = g_slab_rows(BM, BN), LDZ = BN + 4, NT = NW * 64;
  constexpr int TC = GATED ? BN / 8 : BN / 4;  // threads side by side
  static_assert(NT % TC == 0, "a thread keeps its columns");
  const GEpi& e = p.e;
  const int tc = threadIdx.x % TC, tr = threadIdx.x / TC;
  const int zc = GATED ? (tc >> 2) * 32 + (tc & 3) * 4 : tc * 4;  // column of the tile (gated: of the gate)
  const int n = GATED ? bcol + tc * 4 : n0 + zc;                  // column of the result (of a half)
  const bool in_n = n < (GATED ? e.halfp : p.N);
  GCols ec;
  if constexpr (!SPLIT) ec = Epi::cols(e, in_n ? n : 0);
  float cs[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  // what a slab needs beside z is in flight while the slab before is written
  constexpr int STEP = NT / TC, RPT = SR / STEP;  // a thread's rows of a slab
  float res[RPT][4];
  auto load = [&](int s0) {
    if constexpr (!SPLIT) {
      if (in_n) {
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          const int64_t m = m0 + s0 + tr + i * STEP;
          Epi::load(e, ec, m < p.M ? m : p.M - 1, res[i]);
        }
      }
    }
  };
  load(0);
#pragma unroll
  for (int s0 = 0; s0 < BM; s0 += SR) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int row = wm * WM + 16 * i - s0;  // whole 16-row blocks lie in one slab
      if (row >= 0 && row < SR) {
#pragma unroll
        for (int j = 0; j < NI; ++j)
          *reinterpret_cast<f32x4*>(zt + (row + c) * LDZ + wn * WN + 16 * j + 4 * g) = acc[i][j];
      }
    }
    float cur[RPT][4];
#pragma unroll
    for (int i = 0; i < RPT; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) cur[i][v] = res[i][v];
    if (s0 + SR < BM) load(s0 + SR);
    __syncthreads();
    if constexpr (SPLIT) {
      if (in_n) {
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          const int r = tr + i * STEP;
          const int64_t m = m0 + s0 + r;
          if (m >= p.M) break;
          float* part = e.part + ((int64_t)blockIdx.y * p.M + m) * e.ld_part + n;
          *reinterpret_cast<f32x4*>(part) = *reinterpret_cast<const f32x4*>(zt + r * LDZ + zc);
          if constexpr (GATED)
            *reinterpret_cast<f32x4*>(part + e.parth) = *reinterpret_cast<const f32x4*>(zt + r * LDZ + zc + 16);
        }
      }
    } else {
      g_by_act<Epi::kAct>(e.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (!in_n) return;
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          const int r = tr + i * STEP;
          const int64_t m = m0 + s0 + r;
          if (m >= p.M) break;
          const f32x4 x = *reinterpret_cast<const f32x4*>(zt + r * LDZ + zc);
          float z[4] = {x[0], x[1], x[2], x[3]};
          if constexpr (GATED) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(zt + r * LDZ + zc + 16);
            float u[4] = {y[0], y[1], y[2], y[3]};
            Epi::template apply<ACT>(e, ec, m, z, u, cur[i]);
            if constexpr (Epi::kColSum) {
#pragma unroll
              for (int v = 0; v < 4; ++v) cs[0][v] += z[v], cs[1][v] += u[v];
            }
          } else {
            Epi::template apply<ACT>(e, ec, m, z, cur[i]);
            if constexpr (Epi::kColSum) {
#pragma unroll
              for (int v = 0; v < 4; ++v) cs[0][v] += z[v];
            }
          }
        }
      });
    }
  }
  if constexpr (Epi::kColSum && !SPLIT) {
    if (e.colsum) {
      // over the threads that share columns, in order
      constexpr int H = GATED ? 2 : 1;
      __syncthreads();
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int v = 0; v < 4; ++v) zt[tr * (H * TC * 4) + h * TC * 4 + tc * 4 + v] = cs[h][v];
      __syncthreads();
      for (int q = threadIdx.x; q < H * TC * 4; q += NT) {
        float s = 0.f;
        for (int w = 0; w < NT / TC; ++w) s += zt[w * (H * TC * 4) + q];
        const int h = q / (TC * 4), col = (GATED ? bcol : n0) + q % (TC * 4);
        if (col < (GATED ? e.half : e.ncol)) e.colsum[im * e.ld_colsum + col + (GATED ? h * e.half : 0)] = s;
      }
    }
  }
}

// Block of (BM / WM) x (BN / WN) waves.
template <bool AKM, bool BKM, int BM, int BN, int BK, int WM, int WN, class Epi, bool SPLIT>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64)
    k_gemm16(const GArgs<uint16_t> p) {
  constexpr int NWM = BM / WM, NWN = BN / WN, NW = NWM * NWN, MI = WM / 16, NI = WN / 16;
  constexpr bool GATED = Epi::kGated;
  typedef GTile<BM, BK, AKM, NW, false> TA;
  typedef GTile<BN, BK, BKM, NW, GATED> TB;
  constexpr int kStage = TA::kBytes + TB::kBytes;
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4, wm = wave / NWN, wn = wave % NWN;
  uint32_t im, in;
  g_tile_of(blockIdx.x, p.tiles_m, p.tiles_n, 8, im, in);
  const int64_t m0 = (int64_t)im * BM;
  const int n0 = (int)in * BN;               // tile column of Z
  const int bcol = GATED ? (int)in * (BN / 2) : n0;  // first column of B that the tile reads
  const uint16_t *ap = p.a.p, *bp = p.b.p;
  uint32_t split = SPLIT ? blockIdx.y : 0;
  if (SPLIT && p.lo_from && split >= p.lo_from) {
    split -= p.lo_from;
    ap += p.lo_a;
    bp += p.lo_b;
  }
  const int64_t k_from = SPLIT ? (int64_t)split * p.k_split : 0;
  const int64_t k_to = SPLIT ? (k_from + p.k_split < p.K ? k_from + p.k_split : p.K) : p.K;
  const int steps = (int)((k_to - k_from + BK - 1) / BK);

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(g_lds_addr(lds));
  TA ta;
  TB tb;
  ta.init(p.a, wave, lane, 0);
  tb.init(p.b, wave, lane, p.e.halfp);

  auto issue = [&](int t) {
    const int64_t k0 = k_from + (int64_t)t * BK, kl = k_to - k0;
    const uint32_t st = lds0 + (t & 1) * kStage;
    const uint32_t sb = st + TA::kBytes;
    if constexpr (AKM) {
      ta.issue(ap + m0 * p.a.ld + k0, 2 * ((p.a.rows - m0 - 1) * p.a.ld + p.a.cols - k0), kl, st, wave);
    } else {
      ta.issue(ap + k0 * p.a.ld + m0, 2 * ((kl - 1) * p.a.ld + p.a.cols - m0), kl, st, wave);
    }
    if constexpr (BKM) {
      tb.issue(bp + (int64_t)bcol * p.b.ld + k0, 2 * ((p.b.rows - bcol - 1) * p.b.ld + p.b.cols - k0), kl, sb, wave);
    } else {
      // rows that B has: its k may end before A's padded one
      const int64_t rl = (p.b.rows < k_to ? p.b.rows : k_to) - k0;
      tb.issue(bp + k0 * p.b.ld + bcol, 2 * ((rl - 1) * p.b.ld + p.b.cols - bcol), rl, sb, wave);
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
    const char* sb = sa + TA::kBytes;
#pragma unroll
    for (int kb = 0; kb < BK / 32; ++kb) {
      uint4 fa[MI], fb[NI];
#pragma unroll
      for (int j = 0; j < NI; ++j) fb[j] = TB::frag(sb, wn * NI + j, kb, c, g);
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[i] = TA::frag(sa, wm * MI + i, kb, c, g);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mfma_bf16(fb[j], fa[i], acc[i][j]);
    }
  }
  g_epilogue<BM, BN, WM, WN, Epi, SPLIT>(p, acc, reinterpret_cast<float*>(lds), im, m0, n0, bcol, wm, wn, c, g);
}

// ---- float32 operands ------------------------------------------------------------
// The same product with each float32 value as the sum of three bfloat16 parts
// (its leading 8 bits, the next 8, the rest) and the six part products of order
// at most two, so a product term is exact to about 2^-23 of itself.  The parts
// are made on the way to LDS: a step's tile is loaded into registers while the
// MFMAs of the step before run.  No scales: any exponent, whatever lies beside
// it.  Three planes of 32 k a step.  VEC: rows are 16-byte aligned and whole
// multiples of four values.
constexpr int kG32K = 32;

// Four values truncated to three parts.
__device__ __forceinline__ void g_parts3(f32x4 x, uint2 (&p)[3]) {
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    uint32_t u[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      u[v] = __float_as_uint(x[v]);
      if (k < 2) x[v] -= __uint_as_float(u[v] & 0xFFFF0000u);
    }
    p[k] = uint2{__builtin_amdgcn_perm(u[1], u[0], 0x07060302u), __builtin_amdgcn_perm(u[3], u[2], 0x07060302u)};
  }
}

__device__ const float g_zeros[4] = {0.f, 0.f, 0.f, 0.f};

template <int BM, bool KM, int NT, bool GATED, bool VEC>
struct GTile32 {
  static constexpr int kPlane = BM * kG32K * 2;      // bytes
  static constexpr int PER = BM * kG32K / 4 / NT;    // groups of four a thread
  static constexpr int ACROSS = KM ? kG32K / 4 : BM / 4;
  static_assert(BM * kG32K / 4 % NT == 0, "whole groups a thread");
  f32x4 x[PER];

  // first: first row (KM) or column; rows and cols as stored; k0, k_to: the step's range
  __device__ __forceinline__ void load(const GOperand<float>& o, int64_t first, int64_t k0, int64_t k_to, int upper,
                                       int half) {
    // group q: its address and how many of its values exist
    auto at = [&](int q, int64_t& left) {
      const int id = threadIdx.x + q * NT, r = id / ACROSS, s = id % ACROSS * 4;
      int64_t row, col, to;
      if constexpr (KM) {
        row = first + r;
        col = k0 + s;
        to = row < o.rows ? (k_to < o.cols ? k_to : o.cols) : 0;
      } else {
        const int gr = s >> 4;
        row = k0 + r;
        // gated: 16 columns of each half in turn; `half` columns in each
        const int64_t f = first + (GATED ? (gr >> 1) * 16 + (s & 15) : s);
        col = f + (GATED ? (gr & 1) * upper : 0);
        const int64_t wide = GATED ? half + (gr & 1) * upper : o.cols;
        to = row < k_to && row < o.rows ? wide : 0;
      }
      left = to - col;
      return o.p + row * o.ld + col;
    };
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      int64_t left;
      const float* p = at(q, left);
      if (VEC) {
        x[q] = left > 0 ? *reinterpret_cast<const f32x4*>(p) : f32x4{0.f, 0.f, 0.f, 0.f};
      } else {
        // a load of 16 bytes needs 4-byte alignment only; all are issued before the
        // groups at an edge are looked at (gated, 1777 rows, 200 to 2 x 517: 12.4 us,
        // 2.8 more with single floats)
        __builtin_memcpy(&x[q], left >= 4 ? p : g_zeros, 16);
      }
    }
    if constexpr (!VEC) {
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        int64_t left;
        const float* p = at(q, left);
        if (left > 0 && left < 4) {
#pragma unroll
          for (int v = 0; v < 3; ++v)
            if (v < left) x[q][v] = p[v];
        }
      }
    }
  }
  // LDS: KM [row][32], the 16-byte chunk ch of row r at ch ^ ((r >> 1) & 3); k rows as in GTile
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int id = threadIdx.x + q * NT, r = id / ACROSS, s = id % ACROSS;
      uint2 p[3];
      g_parts3(x[q], p);
      char* at = KM ? lds + r * 64 + (((s >> 1) ^ ((r >> 1) & 3)) * 16) + (s & 1) * 8
                    : lds + r * (BM * 2) + (((s >> 2) ^ g_swz<BM>(r)) * 32) + (s & 3) * 8;
#pragma unroll
      for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(at + k * kPlane) = p[k];
    }
  }
  __device__ static __forceinline__ uint4 frag(const char* lds, int i, int c, int g) {
    if constexpr (KM) {
      const int row = 16 * i + c;
      return *reinterpret_cast<const uint4*>(lds + row * 64 + ((g ^ ((c >> 1) & 3)) * 16));
    } else {
      return GTile<BM, kG32K, false, 1, false>::frag(lds, i, 0, c, g);
    }
  }
};

template <bool AKM, bool BKM, int BM, int BN, int WM, int WN, class Epi, bool SPLIT, bool VEC>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64)
    k_gemm32(const GArgs<float> p) {
  constexpr int NWN = BN / WN, NT = (BM / WM) * NWN * 64, MI = WM / 16, NI = WN / 16;
  constexpr bool GATED = Epi::kGated;
  typedef GTile32<BM, AKM, NT, false, VEC> TA;
  typedef GTile32<BN, BKM, NT, GATED, VEC> TB;
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4, wm = wave / NWN, wn = wave % NWN;
  uint32_t im, in;
  g_tile_of(blockIdx.x, p.tiles_m, p.tiles_n, 8, im, in);
  const int64_t m0 = (int64_t)im * BM;
  const int n0 = (int)in * BN, bcol = GATED ? (int)in * (BN / 2) : n0;
  const int64_t k_from = SPLIT ? (int64_t)blockIdx.y * p.k_split : 0;
  const int64_t k_to = SPLIT ? (k_from + p.k_split < p.K ? k_from + p.k_split : p.K) : p.K;
  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  TA ta;
  TB tb;
  ta.load(p.a, m0, k_from, k_to, 0, 0);
  tb.load(p.b, bcol, k_from, k_to, p.e.halfp, p.e.half);
  for (int64_t k0 = k_from; k0 < k_to; k0 += kG32K) {
    __syncthreads();
    ta.store(lds);
    tb.store(lds + 3 * TA::kPlane);
    __syncthreads();
    if (k0 + kG32K < k_to) {
      ta.load(p.a, m0, k0 + kG32K, k_to, 0, 0);
      tb.load(p.b, bcol, k0 + kG32K, k_to, p.e.halfp, p.e.half);
    }
    uint4 fa[3][MI], fb[3][NI];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[k][i] = TA::frag(lds + k * TA::kPlane, wm * MI + i, c, g);
#pragma unroll
      for (int j = 0; j < NI; ++j) fb[k][j] = TB::frag(lds + 3 * TA::kPlane + k * TB::kPlane, wn * NI + j, c, g);
    }
    // the smallest part products first
    constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
    for (int s = 0; s < 6; ++s)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mfma_bf16(fb[pb[s]][j], fa[pa[s]][i], acc[i][j]);
  }
  g_epilogue<BM, BN, WM, WN, Epi, SPLIT>(p, acc, reinterpret_cast<float*>(lds), im, m0, n0, bcol, wm, wn, c, g);
}

// ---- backward of narrow float32 rows --------------------------------------------
// dz, dX and dW of a linear map with both widths up to 128 in one pass over very
// many rows: x and dy are read once, dX written once and dz never leaves the CU
// (three products by tiles read and write it and x again: 2.3 times the bytes).
// A block of eight waves takes tiles of 32 rows; each wave keeps its columns of W
// and of W^T in registers, as three bfloat16 parts.  A tile's x and dz lie in LDS
// in one layout [row][128], which serves as rows of k and, through the
// transposing reads, as k rows:
//   z  = x W       x rows of k,  W k rows        wave w: columns 16 w of z
//   dx = dz W^T    dz rows of k, W rows of k     wave w: columns 16 w of dx
//   dW += x^T dz   x k rows,     dz k rows       a wave: 64 x 32, kept over the tiles
// z of a tile and dx and dW of the one before lie between the same two barriers,
// so one wave's activation runs beside another's products.  120 KB of LDS and
// 256 registers: one block a CU.
constexpr int kNarrow = 128, kNarrowRows = 32;
constexpr int kNarrowThreads = 512;
constexpr int kNarrowPlaneW = kNarrow * kNarrow * 2, kNarrowPlaneR = kNarrowRows * kNarrow * 2;  // bytes
constexpr int kNarrowTile = 3 * kNarrowPlaneR;
constexpr size_t kNarrowLds = 5 * (size_t)kNarrowTile;  // three tiles of x, two of dz; W before them
static_assert(kNarrowLds >= 3 * (size_t)kNarrowPlaneW, "W fits");

struct GNarrow {
  const float *x, *w, *dy, *bias;
  float* dx;
  int64_t ld_x, ld_dy, ld_dx, n;
  int32_t d, f, act;
  float *part, *colsum;  // [blocks][d][ld_part], [blocks][f] (or null)
  int32_t ld_part;
};

// Address of (row, col) in a plane of 256-byte rows: the 32-byte granule is
// swizzled by the rows that a half wave of transposing reads touches (0-3 and
// 8-11 of eight), its halves by the row's bit that is left, so that 16 rows'
// 16-byte reads fall on all banks too.
__device__ __forceinline__ int n_at(int row, int col) {
  return row * 256 + ((col >> 4) ^ ((row & 3) | ((row >> 3 & 1) << 2))) * 32 + ((col >> 3 ^ row >> 2) & 1) * 16 + (col & 7) * 2;
}
// Eight k of row `row`.
__device__ __forceinline__ uint4 n_row8(const char* plane, int row, int k) {
  return *reinterpret_cast<const uint4*>(plane + n_at(row, k));
}
// Rows k0 + 8 g .. + 7 of column 16 blk + c.
__device__ __forceinline__ uint4 n_col8(const char* plane, int k0, int blk, int c, int g) {
  typedef __attribute__((address_space(3))) g_s16x4* lds_ptr;
  const int row = k0 + 8 * g + (c >> 2), col = 16 * blk + 4 * (c & 3);
  const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(plane + n_at(row, col))));
  const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(plane + n_at(row + 4, col))));
  return uint4{a.x, a.y, b.x, b.y};
}
__device__ __forceinline__ void n_put(char* planes, int plane_bytes, int row, int col, f32x4 x) {
  uint2 p[3];
  g_parts3(x, p);
  const int at = n_at(row, col);
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(planes + k * plane_bytes + at) = p[k];
}

// 32 rows x 16 columns over KB blocks of 32 k: the next block's fragments are read
// while the MFMAs of one run.
template <int KB>
__device__ __forceinline__ void n_product(f32x4 (&acc)[2], const uint4 (&fw)[KB][3], const char* planes, int c, int g) {
  constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};  // the smallest part products first
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    uint4 fa[3][2];
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) fa[k][i] = n_row8(planes + k * kNarrowPlaneR, 16 * i + c, 32 * kb + 8 * g);
#pragma unroll
    for (int s = 0; s < 6; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i] = mfma_bf16(fw[kb][pb[s]], fa[pa[s]][i], acc[i]);
  }
}

// KB: blocks of 32 that cover both widths.
template <int KB>
__global__ void __launch_bounds__(kNarrowThreads, 2) k_narrow_bwd(const GNarrow p) {
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4, wm = wave >> 2, wn = wave & 3;
  constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pb[6] = {0, 2, 1, 0, 1, 0};  // the smallest part products first
  const f32x4 zero{0.f, 0.f, 0.f, 0.f};
  for (int id = threadIdx.x; id < kNarrow * kNarrow / 4; id += kNarrowThreads) {
    const int row = id / 32, col = id % 32 * 4;
    n_put(lds, kNarrowPlaneW, row, col,
          row < p.d && col < p.f ? *reinterpret_cast<const f32x4*>(p.w + (int64_t)row * p.f + col) : zero);
  }
  const int zc = 16 * wave + 4 * g;  // this lane's columns of z and of dx
  float b[4], cs[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int v = 0; v < 4; ++v) b[v] = p.bias && zc < p.f ? p.bias[zc + v] : 0.f;
  f32x4 dw[4][2];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) dw[i][j] = zero;

  // the next tile's rows are in flight during this one
  const int64_t tiles = (p.n + kNarrowRows - 1) / kNarrowRows;
  f32x4 xr[2], dyr[2];
  auto load_x = [&](int64_t t) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int id = threadIdx.x + q * kNarrowThreads, col = id % 32 * 4;
      const int64_t row = t * kNarrowRows + id / 32;
      const bool in = row < p.n && col < p.d;
      xr[q] = *reinterpret_cast<const f32x4*>(p.x + (in ? row * p.ld_x + col : 0));
      if (!in) xr[q] = zero;
    }
  };
  auto load_dy = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t row = t * kNarrowRows + 16 * i + c;
      const bool in = row < p.n && zc < p.f;
      dyr[i] = *reinterpret_cast<const f32x4*>(p.dy + (in ? row * p.ld_dy + zc : 0));
      if (!in) dyr[i] = zero;
    }
  };
  // this wave's columns of W and of W^T, to registers
  __syncthreads();
  uint4 wz[KB][3], wx[KB][3];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      wz[kb][k] = n_col8(lds + k * kNarrowPlaneW, 32 * kb, wave, c, g);
      wx[kb][k] = n_row8(lds + k * kNarrowPlaneW, 16 * wave + c, 32 * kb + 8 * g);
    }
  __syncthreads();
  auto put_x = [&](int at) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int id = threadIdx.x + q * kNarrowThreads;
      n_put(lds + at * kNarrowTile, kNarrowPlaneR, id / 32, id % 32 * 4, xr[q]);
    }
  };
  const int64_t step = gridDim.x;
  load_x(blockIdx.x);
  load_dy(blockIdx.x);
  put_x(0);
  load_x(blockIdx.x + step);
  int bx = 0, bz = 0;  // buffers of this tile
  for (int64_t t = blockIdx.x; t < tiles + step; t += step) {
    const int px = bx == 0 ? 2 : bx - 1, pz = bz ^ 1, nx = bx == 2 ? 0 : bx + 1;  // of the tile before, of the next one
    __syncthreads();
    const char* lx = lds + bx * kNarrowTile;
    f32x4 z[2] = {zero, zero};
    if (t < tiles && p.act != HG_ACT_NONE && 16 * wave < p.f) n_product<KB>(z, wz, lx, c, g);
    if (t < tiles) {
      // dz
      char* lz = lds + (3 + bz) * kNarrowTile;
      g_by_act<true>(p.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float y[4], f[4], s[4];
#pragma unroll
          for (int v = 0; v < 4; ++v) y[v] = z[i][v] + b[v];
          g_act4<ACT, true>(y, f, s);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            y[v] = dyr[i][v] * s[v];  // zero in rows and columns that are not there
            cs[v] += y[v];
          }
          n_put(lz, kNarrowPlaneR, 16 * i + c, zc, f32x4{y[0], y[1], y[2], y[3]});
        }
      });
      load_dy(t + step);
    }
    put_x(nx);
    load_x(t + 2 * step);
    if (t >= step) {
      const char *lq = lds + px * kNarrowTile, *lz = lds + (3 + pz) * kNarrowTile;
      // dX
      if (16 * wave < p.d) {
        f32x4 o[2] = {zero, zero};
        n_product<KB>(o, wx, lz, c, g);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int64_t row = (t - step) * kNarrowRows + 16 * i + c;
          if (row < p.n && zc < p.d) *reinterpret_cast<f32x4*>(p.dx + row * p.ld_dx + zc) = o[i];
        }
      }
      // dW
      if (64 * wm < p.d && 32 * wn < p.f) {
        uint4 fz[3][2];
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int j = 0; j < 2; ++j) fz[k][j] = n_col8(lz + k * kNarrowPlaneR, 0, 2 * wn + j, c, g);
#pragma unroll
        for (int i0 = 0; i0 < 4; i0 += 2) {
          uint4 fx[3][2];
#pragma unroll
          for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) fx[k][i] = n_col8(lq + k * kNarrowPlaneR, 0, 4 * wm + i0 + i, c, g);
#pragma unroll
          for (int s = 0; s < 6; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 2; ++j) dw[i0 + i][j] = mfma_bf16(fz[pb[s]][j], fx[pa[s]][i], dw[i0 + i][j]);
        }
      }
    }
    bx = nx;
    bz ^= 1;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = 64 * wm + 16 * i + c;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = 32 * wn + 16 * j + 4 * g;
      if (m < p.d && n < p.f)
        *reinterpret_cast<f32x4*>(p.part + ((int64_t)blockIdx.x * p.d + m) * p.ld_part + n) = dw[i][j];
    }
  }
  if (p.colsum) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) cs[v] += __shfl_xor(cs[v], o, 64);
      if (c == 0 && zc < p.f) p.colsum[(int64_t)blockIdx.x * p.f + zc + v] = cs[v];
    }
  }
}

// Sum of the splits, then the epilogue.  SL threads share the splits of four
// columns of a row (each every SL-th in order, then the SL sums in order).
template <class Epi, int SL>
__global__ void __launch_bounds__(256) k_product_join(const GShape p, int splits) {
  constexpr int QB = 256 / SL, H = Epi::kGated ? 2 : 1;
  __shared__ f32x4 sh[SL > 1 ? SL : 1][H][SL > 1 ? QB : 1];
  const GEpi& e = p.e;
  const int cols = Epi::kGated ? e.halfp : p.N, quads = (cols + 3) / 4;
  const int q = threadIdx.x % QB, sl = threadIdx.x / QB;
  const int64_t id = (int64_t)blockIdx.x * QB + q, m = id / quads;
  const bool in = m < p.M;
  const int n = (int)(id - m * quads) * 4;
  f32x4 s[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!in) continue;
    const float* at = e.part + m * e.ld_part + n + h * e.parth;
#pragma unroll 8
    for (int k = sl; k < splits; k += SL) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(at + (int64_t)k * p.M * e.ld_part);
#pragma unroll
      for (int v = 0; v < 4; ++v) s[h][v] += x[v];
    }
  }
  if constexpr (SL > 1) {
#pragma unroll
    for (int h = 0; h < H; ++h) sh[sl][h][q] = s[h];
    __syncthreads();
    if (sl > 0) return;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int k = 1; k < SL; ++k) {
        const f32x4 x = sh[k][h][q];
#pragma unroll
        for (int v = 0; v < 4; ++v) s[h][v] += x[v];
      }
  }
  if (!in) return;
  float z[4] = {s[0][0], s[0][1], s[0][2], s[0][3]}, r[4];
  const GCols ec = Epi::cols(e, n);
  Epi::load(e, ec, m, r);
  g_by_act<Epi::kAct>(e.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if constexpr (Epi::kGated) {
      float u[4] = {s[H - 1][0], s[H - 1][1], s[H - 1][2], s[H - 1][3]};
      Epi::template apply<ACT>(e, ec, m, z, u, r);
    } else {
      Epi::template apply<ACT>(e, ec, m, z, r);
    }
  });
}

}  // namespace hg
