// Linear attention with a decay for each head.
//
//   S_t = l S_{t-1} + k_t^T v_t,   o_t = scale q_t S_t,   l = exp(log_decay[h])
//
// A sequence is walked in chunks of C tokens.  With S the state before a
// chunk and i, j its tokens,
//   o_i = sum_{j <= i} l^(i-j) (q_i . k_j) v_j + l^(i+1) q_i S
//   S'  = l^n S + sum_j l^(n-1-j) k_j^T v_j            (n tokens in the chunk)
// so everything is matrix products on the MFMA.  Only non-negative powers of
// l are formed: no decay overflows.
//
// The backward is the same walk with the roles changed (R is the gradient of
// the state, walked from the last token):
//   dq = scan(q := do, k := v, v := k)        its state is S^T
//   dk = reverse scan(q := v, k := do, v := q)  its state is R^T
//   dv = reverse scan(q := k, k := q, v := do)  its state is R
// A reverse walk adds a token's k^T v before the decay, so its powers are
// l^i and l^(n-j) instead of l^(i+1) and l^(n-1-j): the `lead` of 1.
//
// Work split: a block takes one head of one sequence, or one segment of it
// when there are too few of those to fill the chip.  Then a first pass forms
// every segment's sum, a second adds them up along the sequence, and the walk
// starts each segment from its state.  The backward's three walks are one
// launch; dk takes dv's segment states transposed.  Where query heads share key
// heads, a block of the backward takes two of them in turn for every chunk, so
// the sum of their dk and dv stays in registers and what they share is loaded
// once (8 x 2048 tokens, 16 heads on 8, d = 64: 98 to 105 us, 131 with one float32
// gradient a query head and a pass that adds them).
//
// A chunk is 32 tokens: half of the registers and LDS of 64, so that a CU holds
// 16 waves (133 us and 121 for the same backward with one head a block).  The
// powers of the decay that a chunk needs are a table in LDS.
//
// Layout: a wave owns 16 columns of v, of the state and of o and all rows; q, k
// and v tiles and P, whose blocks the waves share out, pass through LDS.  With
// the tiles' operands taken as blocks of 16 values, 4 g .. 4 g + 3 in lane group g, every product's
// result lies as the next product's operand needs it:
//   P^T = K Q^T       lane (c, g): keys 4 g + v of query c    (operand of V^T P^T)
//   S  += K^T (w V)   lane (c, g): rows 4 g + v of column c   (operand of S^T Q^T)
//   O^T = S^T Q^T + V^T P^T   lane (c, g): columns 4 g + v of token c
// so S never leaves the wave's registers.
//
// Precision: sums, states and decays are float32.  float32 calls use the
// float32 MFMA.  In bfloat16 calls q, k and v enter exactly, P and the copy of
// S that multiplies q as a bfloat16 value and the rest of it (2^-17), and the
// state takes w V in three bfloat16 parts (2^-24): what remains is the one
// rounding of o.
#include "hg_mfma.h"

namespace hg {
namespace {

constexpr int kMaxD = 128;
constexpr int kChunk = 32;              // tokens of a step
constexpr int64_t kMaxToken = 1 << 22;  // token stride: a chunk stays below 2^31 bytes

// One operand: element (sequence b, token t, head h, column x) at
// p[b * sb + t * st + (h / hdiv) * sh + x].
struct Role {
  const void* p;
  int64_t sb, st, sh;
  int32_t hdiv;
};

struct Walk {
  Role q, k, v, o;
  const float* log_decay;
  const int32_t* lens;     // tokens of each sequence, or null
  const float* s_in;       // [B][H][d][d] state before the walk, or null
  float* s_out;            // state after it, or null
  float* seg;              // segment sums, then states before each segment
  int64_t T;
  int64_t seg_len;         // a multiple of the chunk
  int32_t segs, H, d;
  int32_t reverse;         // walk from the last token; 1: its lead too
  int32_t s_trans;         // the walk's state is the transpose of s_in and s_out
  int32_t seg_trans;       // ... and of seg (another walk's)
  int32_t f32_out;         // o is float32 whatever the operands are
  int32_t sum_o;           // o is the sum over a block's heads, which share q; else they share k and v
  float kv_scale, o_scale;
};

// The walks of a call, one a blockIdx.z.
struct Walks {
  Walk w[3];
};

typedef __bf16 l_bf16x4 __attribute__((ext_vector_type(4)));
typedef short l_s16x4 __attribute__((ext_vector_type(4)));

// Sixteen values of a contraction, four a lane.
template <class T>
struct Blk;
template <>
struct Blk<float> {
  typedef f32x4 type;
  static __device__ __forceinline__ type zero() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ type of(f32x4 x) { return x; }
};
template <>
struct Blk<bf16_t> {
  typedef uint2 type;
  static __device__ __forceinline__ type zero() { return uint2{0u, 0u}; }
  // rounded to nearest
  static __device__ __forceinline__ type of(f32x4 x) {
    return __builtin_bit_cast(uint2, __builtin_convertvector(x, l_bf16x4));
  }
};
__device__ __forceinline__ f32x4 wide(f32x4 x) { return x; }
__device__ __forceinline__ f32x4 wide(uint2 x) {
  return f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u), __uint_as_float(x.y << 16),
               __uint_as_float(x.y & 0xFFFF0000u)};
}

// A float32 factor of a product: as it is, or its bfloat16 value and the rest
// of it (16 bits in all).
template <class T>
struct Factor {
  static constexpr int N = sizeof(T) == 4 ? 1 : 2;
  typename Blk<T>::type x[N];
  __device__ __forceinline__ void set(f32x4 v) {
    x[0] = Blk<T>::of(v);
    if constexpr (N == 2) {
      const f32x4 h = wide(x[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = v[i] - h[i];
      x[1] = Blk<T>::of(v);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = Blk<T>::zero();
  }
};

// Element i of the factor of a lane.
template <class T>
__device__ __forceinline__ float element(const Factor<T>& f, int i) {
  float s = 0.f;
#pragma unroll
  for (int x = Factor<T>::N - 1; x >= 0; --x) {
    const f32x4 w = wide(f.x[x]);
    s += i == 0 ? w[0] : i == 1 ? w[1] : i == 2 ? w[2] : w[3];
  }
  return s;
}

// The values with zero in the place of infinities and NaN.
__device__ __forceinline__ f32x4 finite(f32x4 x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = fabsf(x[i]) < INFINITY ? x[i] : 0.f;
  return x;
}
__device__ __forceinline__ uint2 finite(uint2 x) { return Blk<bf16_t>::of(finite(wide(x))); }

// acc += A B over 32 values
__device__ __forceinline__ f32x4 mma32(uint2 a0, uint2 a1, uint2 b0, uint2 b1, f32x4 acc) {
  return mfma_bf16(uint4{a0.x, a0.y, a1.x, a1.y}, uint4{b0.x, b0.y, b1.x, b1.y}, acc);
}
__device__ __forceinline__ f32x4 mma32(f32x4 a0, f32x4 a1, f32x4 b0, f32x4 b1, f32x4 acc) {
#pragma unroll
  for (int v = 0; v < 4; ++v) acc = mfma4(a0[v], b0[v], acc);
#pragma unroll
  for (int v = 0; v < 4; ++v) acc = mfma4(a1[v], b1[v], acc);
  return acc;
}

// acc += A B over 16 values
__device__ __forceinline__ f32x4 mma16(uint2 a, uint2 b, f32x4 acc) {
  return mma32(a, uint2{0u, 0u}, b, uint2{0u, 0u}, acc);
}
__device__ __forceinline__ f32x4 mma16(f32x4 a, f32x4 b, f32x4 acc) {
#pragma unroll
  for (int v = 0; v < 4; ++v) acc = mfma4(a[v], b[v], acc);
  return acc;
}

// COLS: k and v, read down columns; else q, read along rows.
template <class T, int DP, bool COLS>
struct Tile {
  static constexpr int EL = Elt<T>::EL;
  // 16 bytes more than the row, and 32 for bfloat16 rows whose transposing reads
  // take 8 rows of 32 bytes a half wave: what one read touches falls on all banks
  // (16 heads of 16381 tokens, d = 128: 127 us, 133 with 32 for all)
  static constexpr int LD = DP + (sizeof(T) == 4 ? 4 : COLS ? 16 : 8);
  typedef typename Blk<T>::type B;
  // 16 columns of row r: lane's four
  static __device__ __forceinline__ B row4(const T* t, int r, int blk, int g) {
    return *reinterpret_cast<const B*>(t + r * LD + 16 * blk + 4 * g);
  }
  // 32 columns of row r: lane's eight, 8 g .. (float32: four and four of two blocks)
  static __device__ __forceinline__ void row8(const T* t, int r, int blk, int g, B& x, B& y) {
    if constexpr (sizeof(T) == 2) {
      const uint4 w = *reinterpret_cast<const uint4*>(t + r * LD + 16 * blk + 8 * g);
      x = uint2{w.x, w.y};
      y = uint2{w.z, w.w};
    } else {
      x = row4(t, r, blk, g);
      y = row4(t, r, blk + 1, g);
    }
  }
  // rows 16 rb + 4 g .. + 3 of column 16 cb + c
  static __device__ __forceinline__ B col4(const T* t, int rb, int cb, int c, int g) {
    if constexpr (sizeof(T) == 4) {
      const T* p = t + (16 * rb + 4 * g) * LD + 16 * cb + c;
      return f32x4{p[0], p[LD], p[2 * LD], p[3 * LD]};
    } else {
      typedef __attribute__((address_space(3))) l_s16x4* lds_ptr;
      const T* p = t + (16 * rb + 4 * g + (c >> 2)) * LD + 16 * cb + 4 * (c & 3);
      return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p)));
    }
  }
};

// Tokens of sequence b.
__device__ __forceinline__ int64_t len_of(const int32_t* lens, int b, int64_t T) {
  if (!lens) return T;
  const int64_t l = lens[b];
  return l < 0 ? 0 : (l > T ? T : l);
}

// -infinity (a head that keeps nothing) as a number: its powers are 1, 0, 0, ...
__device__ __forceinline__ float log_of(float x) { return x < -1e30f ? -1e30f : x; }

// Power n >= 0 of the decay: exp(n log l), 1 for n = 0 whatever l is.
__device__ __forceinline__ float decay(float lg, int n) { return n <= 0 ? 1.f : expf(lg * (float)n); }

// C rows of one operand: row i holds position u0 + i of the walk (token u0 + i,
// or last - u0 - i in a reverse walk); rows from n on and columns from d on are
// zero.  `load` starts the loads of a chunk, `store` puts it into LDS: the next
// chunk's rows are in flight while the MFMAs of this one run.  Buffer loads: the
// descriptor starts at the chunk's first token and ends with its last, what lies
// outside reads as zero, so no branch holds a load back.
template <class T, int DP, int C, int NT>
struct Rows {
  static constexpr int EL = Elt<T>::EL, CH = DP / EL, N = C * CH / NT;
  static_assert(C * CH % NT == 0, "whole chunks per thread");
  u32x4 x[N];
  int off[N];
  __device__ __forceinline__ void init(int64_t st, int d, bool reverse) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int id = threadIdx.x + q * NT, row = id / CH, col = id % CH * EL;
      off[q] = col < d ? ((reverse ? C - 1 - row : row) * (int)st + col) * (int)sizeof(T) : 0x7FFFFF00;
    }
  }
  // first: the chunk's first token in memory
  __device__ __forceinline__ void load(const T* first, int64_t st, int n, int d, bool reverse) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(first), 0,
                                                        (int)(((n - 1) * (int)st + d) * (int)sizeof(T)), 0x00020000);
    // a reverse walk's missing rows lie before the first token
    const int back = reverse ? (C - n) * (int)st * (int)sizeof(T) : 0;
#pragma unroll
    for (int q = 0; q < N; ++q) x[q] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off[q] - back, 0, 0);
  }
  template <class TL>
  __device__ __forceinline__ void store(T* lds) const {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int id = threadIdx.x + q * NT, row = id / CH, col = id % CH * EL;
      *reinterpret_cast<u32x4*>(lds + row * TL::LD + col) = x[q];
    }
  }
  // whether any of this thread's values is infinite or NaN
  __device__ __forceinline__ bool not_finite() const {
    bool bad = false;
#pragma unroll
    for (int q = 0; q < N; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
          bad |= (x[q][i] & 0x7F800000u) == 0x7F800000u;
        } else {
          bad |= (x[q][i] & 0x7F80u) == 0x7F80u || (x[q][i] & 0x7F800000u) == 0x7F800000u;
        }
      }
    return bad;
  }
};

// v truncated to three bfloat16 parts (24 bits in all), four values a lane
__device__ __forceinline__ void parts3(f32x4 x, uint2 (&p)[3]) {
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

template <int DP>
struct Shape {
  static constexpr int NB = DP / 16;        // 16-column blocks of a row, a wave each
  static constexpr int THREADS = 64 * NB;
};

// GR heads of one sequence that share their key head, or a segment of them.
// SUMS: only the segment's sum.  Registers for 16 waves a CU, or for 12 and 8 where
// the states of two heads, or six waves a block, leave no use for more (two heads
// at d = 64 spilled 28 bytes a lane at 16: 114 us for the backward of 8 x 2048
// tokens, 98 to 105 at 12; float32 at d = 32 eight registers: 64 x 512 tokens, 8
// heads on 4, 112 us, 101 at 12).
template <class T, int DP, bool SUMS, int GR>
__global__ void __launch_bounds__(Shape<DP>::THREADS, GR == 2 && DP > 64 ? 2 : DP == 96 || (GR == 2 && DP * sizeof(T) >= 128) ? 3 : 4) k_linattn_scan(const Walks walks) {
  const Walk& a = walks.w[blockIdx.z];
  constexpr int NB = Shape<DP>::NB, NTHR = Shape<DP>::THREADS, C = kChunk, RB = C / 16;
  typedef Tile<T, DP, true> TL;
  typedef Tile<T, DP, false> TQ;
  typedef typename Blk<T>::type B;
  constexpr bool kF32 = sizeof(T) == 4;
  constexpr int NP = RB * (RB + 1) / 2;  // 16 x 16 blocks of P on and below the diagonal
  __shared__ __align__(16) T lk[C * TL::LD];
  __shared__ __align__(16) T lv[C * TL::LD];
  __shared__ __align__(16) T lq[SUMS ? 16 : C * TQ::LD];
  __shared__ __align__(16) Factor<T> lp[SUMS ? 1 : NP][64];
  __shared__ float pw[GR][C + 1];  // powers of the heads' decays
  __shared__ int bad_v;            // the last fill of lv that held an infinity or a NaN
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int hb = a.H / GR, h = blockIdx.x % hb * GR, b = blockIdx.x / hb, seg = blockIdx.y;
  const int d = a.d;
  const bool sum_o = GR > 1 && a.sum_o;
  // positions fit 32 bits (T < 2^31); addresses are formed in 64
  const int L = (int)len_of(a.lens, b, a.T);
  const int u_from = (int)((int64_t)seg * a.seg_len), u_end = (int)(u_from + a.seg_len < a.T ? u_from + a.seg_len : a.T);
  const int u_to = u_end < L ? u_end : L;
  const int lead = a.reverse ? 1 : 0;
  const T* kp = static_cast<const T*>(a.k.p) + b * a.k.sb + (h / a.k.hdiv) * a.k.sh;
  const T* vp = static_cast<const T*>(a.v.p) + b * a.v.sb + (h / a.v.hdiv) * a.v.sh;
  const T* qp = SUMS ? nullptr : static_cast<const T*>(a.q.p) + b * a.q.sb + (h / a.q.hdiv) * a.q.sh;
  const int osz = kF32 || a.f32_out ? 4 : 2;
  char* op = SUMS ? nullptr : static_cast<char*>(const_cast<void*>(a.o.p)) + (b * a.o.sb + (h / a.o.hdiv) * a.o.sh) * osz;
  // from a head to the next: the operand that the block's heads do not share
  const int64_t q_head = sum_o ? 0 : a.q.sh, k_head = sum_o ? a.k.sh : 0, v_head = sum_o ? a.v.sh : 0;
  const int64_t bh = (int64_t)b * a.H + h;  // of the first head
  const float po = a.kv_scale * a.o_scale;

  if constexpr (!SUMS) {
    // tokens past the sequence's end: zero rows
    const int z0 = u_from > L ? u_from : L, ch = d / 4;
    for (int r = 0; r < (sum_o ? 1 : GR); ++r)
      for (int64_t i = threadIdx.x; i < (int64_t)(u_end - z0) * ch; i += NTHR) {
        char* p = op + ((z0 + i / ch) * a.o.st + r * a.o.sh + i % ch * 4) * osz;
        if (osz == 4) {
          *reinterpret_cast<f32x4*>(p) = f32x4{0.f, 0.f, 0.f, 0.f};
        } else {
          *reinterpret_cast<uint2*>(p) = uint2{0u, 0u};
        }
      }
    if (u_from >= L && seg > 0) return;  // segment 0 of an empty sequence still hands its state on
  } else {
    if (u_from >= L) return;
  }

  for (int i = threadIdx.x; i < GR * (C + 1); i += NTHR) pw[i / (C + 1)][i % (C + 1)] = decay(log_of(a.log_decay[h + i / (C + 1)]), i % (C + 1));

  // state: rows 16 i + 4 g + v, columns 16 wave + c
  f32x4 S[GR][NB];
  float* seg_at = a.seg ? a.seg + ((bh * a.segs + seg) * (NB * NB)) * 256 : nullptr;
  const int64_t seg_head = (int64_t)a.segs * (NB * NB * 256);  // from a head's states to the next one's
#pragma unroll
  for (int r = 0; r < GR; ++r)
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      f32x4& x = S[r][i];
      x = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (!SUMS) {
        if (a.segs > 1) {
          const float* at = seg_at + r * seg_head;
          if (!a.seg_trans) {
            x = *reinterpret_cast<const f32x4*>(at + (i * NB + wave) * 256 + lane * 4);
          } else {
            // element (r, c) of the block lies where (c, r) of the mirrored block does
#pragma unroll
            for (int v = 0; v < 4; ++v)
              x[v] = at[(wave * NB + i) * 256 + ((c >> 2) * 16 + 4 * g + v) * 4 + (c & 3)];
          }
        } else if (a.s_in) {
          const int col = 16 * wave + c;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int row = 16 * i + 4 * g + v;
            if (row < d && col < d) x[v] = a.s_in[(bh + r) * d * d + (a.s_trans ? col * d + row : row * d + col)];
          }
        }
      }
    }

  Rows<T, DP, C, NTHR> rk, rv, rq;
  rk.init(a.k.st, d, a.reverse);
  rv.init(a.v.st, d, a.reverse);
  if constexpr (!SUMS) rq.init(a.q.st, d, a.reverse);
  auto load = [&](int u0, int r) {
    const int n = u_to - u0 < C ? u_to - u0 : C;
    const int64_t t = a.reverse ? L - n - u0 : u0;
    if (r == 0 || sum_o) {
      rk.load(kp + t * a.k.st + r * k_head, a.k.st, n, d, a.reverse);
      rv.load(vp + t * a.v.st + r * v_head, a.v.st, n, d, a.reverse);
    }
    if constexpr (!SUMS)
      if (r == 0 || !sum_o) rq.load(qp + t * a.q.st + r * q_head, a.q.st, n, d, a.reverse);
  };
  // this lane's columns of o in row c of a block of 16
  const uint32_t o_off = SUMS ? 0 : (uint32_t)(((a.reverse ? 15 - c : c) * (int)a.o.st + 16 * wave + 4 * g) * osz);

  f32x4 sum[RB];  // o of the block's heads so far
  int fill = 0;   // of lv
  if (threadIdx.x == 0) bad_v = 0;
  if (u_from < u_to) load(u_from, 0);
  for (int u0 = u_from; u0 < u_to; u0 += C) {
    const int n = u_to - u0 < C ? u_to - u0 : C;
#pragma unroll
    for (int hr = 0; hr < GR; ++hr) {
      __syncthreads();
      if (hr == 0 || sum_o) {
        rk.template store<TL>(lk);
        rv.template store<TL>(lv);
        ++fill;
        if constexpr (!SUMS)
          if (rv.not_finite()) bad_v = fill;
      }
      if constexpr (!SUMS)
        if (hr == 0 || !sum_o) rq.template store<TQ>(lq);
      __syncthreads();
      if (hr + 1 < GR) {
        load(u0, hr + 1);
      } else if (u0 + C < u_to) {
        load(u0 + C, 0);
      }
      if constexpr (!SUMS) {
        // P, its blocks shared out over the waves
        for (int pr = wave; pr < NP; pr += NB) {
          const int r = pr >= 1 ? 1 : 0, kt = pr - r;
          f32x4 s{0.f, 0.f, 0.f, 0.f}, s1{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < NB; i += 2) {
            B k0, k1, q0, q1;
            if (i + 1 < NB) {
              TL::row8(lk, 16 * kt + c, i, g, k0, k1);
              TQ::row8(lq, 16 * r + c, i, g, q0, q1);
            } else {
              k0 = TL::row4(lk, 16 * kt + c, i, g);
              q0 = TQ::row4(lq, 16 * r + c, i, g);
              k1 = q1 = Blk<T>::zero();
            }
            f32x4& acc = (i & 2) ? s1 : s;  // two chains
            acc = i + 1 < NB ? mma32(k0, k1, q0, q1, acc) : mma16(k0, q0, acc);
          }
#pragma unroll
          for (int v = 0; v < 4; ++v) s[v] += s1[v];
          const int x = 16 * (r - kt) + c - 4 * g;  // tokens from key 4 g to the query
#pragma unroll
          for (int v = 0; v < 4; ++v) s[v] = x >= v ? s[v] * (pw[hr][x >= v ? x - v : 0] * po) : 0.f;
          Factor<T> f;
          f.set(s);
          lp[pr][lane] = f;
        }
        // q S, the chains of the rows side by side
        f32x4 o[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) o[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NB; i += 2) {
          const bool two = i + 1 < NB;
          B q0[RB], q1[RB];
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            q0[r] = TQ::row4(lq, 16 * r + c, i, g);
            q1[r] = two ? TQ::row4(lq, 16 * r + c, two ? i + 1 : i, g) : Blk<T>::zero();
          }
          Factor<T> s0, s1;
          s0.set(S[hr][i]);
          if (two) {
            s1.set(S[hr][two ? i + 1 : i]);
          } else {
            s1.zero();
          }
#pragma unroll
          for (int x = Factor<T>::N - 1; x >= 0; --x)
#pragma unroll
            for (int r = 0; r < RB; ++r)
              o[r] = two ? mma32(s0.x[x], s1.x[x], q0[r], q1[r], o[r]) : mma16(s0.x[x], q0[r], o[r]);
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float rowp = pw[hr][16 * r + c + 1 - lead] * a.o_scale;
#pragma unroll
          for (int v = 0; v < 4; ++v) o[r][v] = sum_o && hr > 0 ? fmaf(o[r][v], rowp, sum[r][v]) : o[r][v] * rowp;
        }
        __syncthreads();
        // P v.  Above the diagonal P is zero, and 0 times an infinity or a NaN is
        // none: those values leave their diagonal block's product and are added for
        // the tokens that they belong to.
        const bool bad = bad_v == fill;
#pragma unroll
        for (int kt = 0; kt < RB; kt += 2) {
          const B v0 = TL::col4(lv, kt, wave, c, g), v1 = TL::col4(lv, kt + 1, wave, c, g);
          B d0 = v0, d1 = v1;
          if (bad) {
            d0 = finite(v0);
            d1 = finite(v1);
          }
#pragma unroll
          for (int r = kt; r < RB; ++r) {
            const Factor<T> p0 = lp[r * (r + 1) / 2 + kt][lane];
            Factor<T> p1 = p0;
            if (r > kt) p1 = lp[r * (r + 1) / 2 + kt + 1][lane];
#pragma unroll
            for (int x = Factor<T>::N - 1; x >= 0; --x)
              o[r] = r > kt ? mma32(v0, d1, p0.x[x], p1.x[x], o[r]) : mma16(d0, p0.x[x], o[r]);
          }
        }
        if (bad) {
          for (int y = 0; y <= c; ++y)
#pragma unroll
            for (int r = 0; r < RB; ++r) {
              const float p = element<T>(lp[r * (r + 3) / 2][16 * (y >> 2) + c], y & 3);
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                const float x = Elt<T>::get(lv + (16 * r + y) * TL::LD + 16 * wave + 4 * g + v);
                if (!(fabsf(x) < INFINITY)) o[r][v] = fmaf(p, x, o[r][v]);
              }
            }
        }
        if (sum_o && hr + 1 < GR) {
#pragma unroll
          for (int r = 0; r < RB; ++r) sum[r] = o[r];
        } else {
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            const int64_t t = a.reverse ? L - 1 - u0 - 16 * r - 15 : u0 + 16 * r;  // token of row 0, or of row 15
            char* p = op + (t * a.o.st + (sum_o ? 0 : hr * a.o.sh)) * osz + o_off;
            if (16 * wave + 4 * g < d && 16 * r + c < n) {
              if (osz == 4) {
                *reinterpret_cast<f32x4*>(p) = o[r];
              } else {
                *reinterpret_cast<uint2*>(p) = Blk<bf16_t>::of(o[r]);
              }
            }
          }
        }
      }

      // state
      const float dn = pw[hr][n];
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) S[hr][i][v] *= dn;
#pragma unroll
      for (int tb = 0; tb < RB; tb += 2) {
        // w v of this wave's columns
        f32x4 w0 = wide(TL::col4(lv, tb, wave, c, g)), w1 = wide(TL::col4(lv, tb + 1, wave, c, g));
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int x = n - 1 + lead - 16 * tb - 4 * g - v;  // (rows past the chunk's end are zero)
          w0[v] *= pw[hr][x > 0 ? x : 0] * a.kv_scale;
          w1[v] *= pw[hr][x > 16 ? x - 16 : 0] * a.kv_scale;
        }
        uint2 p0[3], p1[3];
        if constexpr (!kF32) {
          parts3(w0, p0);
          parts3(w1, p1);
        }
        // chains side by side, at most U blocks' operands at a time
        constexpr int U = NB < 4 ? NB : kF32 ? 2 : 4;
#pragma unroll
        for (int i0 = 0; i0 < NB; i0 += U) {
          B k0[U], k1[U];
#pragma unroll
          for (int i = 0; i < U && i0 + i < NB; ++i) {
            k0[i] = TL::col4(lk, tb, i0 + i, c, g);
            k1[i] = TL::col4(lk, tb + 1, i0 + i, c, g);
          }
#pragma unroll
          for (int x = kF32 ? 0 : 2; x >= 0; --x)
#pragma unroll
            for (int i = 0; i < U && i0 + i < NB; ++i) {
              f32x4& s = S[hr][i0 + i];
              if constexpr (kF32) {
                s = mma32(k0[i], k1[i], w0, w1, s);
              } else {
                s = mma32(k0[i], k1[i], p0[x], p1[x], s);
              }
            }
        }
      }
    }
  }

#pragma unroll
  for (int r = 0; r < GR; ++r) {
    if constexpr (SUMS) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        *reinterpret_cast<f32x4*>(seg_at + r * seg_head + (i * NB + wave) * 256 + lane * 4) = S[r][i];
    } else if (a.segs == 1 && a.s_out) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int col = 16 * wave + c;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int row = 16 * i + 4 * g + v;
          if (row < d && col < d) a.s_out[(bh + r) * d * d + (a.s_trans ? col * d + row : row * d + col)] = S[r][i][v];
        }
      }
    }
  }
}

// The segments' sums added up along each sequence: each becomes the state
// before its segment, the last one's successor the state after the walk.  A
// thread takes four elements (a lane's share of one 16 x 16 block).
template <int DP>
__global__ void __launch_bounds__(256) k_linattn_join(const Walks walks, int64_t bhs) {
  const Walk& a = walks.w[blockIdx.z];
  constexpr int NB = DP / 16, Q = NB * NB * 64;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, bh = id / Q;
  if (bh >= bhs) return;
  const int q = (int)(id - bh * Q), blk = q >> 6, lane = q & 63, c = lane & 15, g = lane >> 4;
  const int h = (int)(bh % a.H), b = (int)(bh / a.H), d = a.d;
  const int64_t L = len_of(a.lens, b, a.T);
  const float lg = log_of(a.log_decay[h]), whole = decay(lg, (int)a.seg_len);
  const int col = 16 * (blk % NB) + c, row = 16 * (blk / NB) + 4 * g;
  f32x4 S{0.f, 0.f, 0.f, 0.f};
  auto at = [&](int v) { return bh * d * d + (a.s_trans ? col * d + row + v : (row + v) * d + col); };
  if (a.s_in && col < d) {
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (row + v < d) S[v] = a.s_in[at(v)];
  }
  float* p = a.seg + bh * a.segs * (int64_t)(NB * NB * 256) + (int64_t)q * 4;
  const int live = (int)((L + a.seg_len - 1) / a.seg_len);
  constexpr int U = 8;  // sums in flight
  for (int s0 = 0; s0 < live; s0 += U) {
    f32x4 x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) x[i] = *reinterpret_cast<const f32x4*>(p + (s0 + i < live ? s0 + i : s0) * (int64_t)(NB * NB * 256));
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int s = s0 + i;
      if (s >= live) break;
      *reinterpret_cast<f32x4*>(p + s * (int64_t)(NB * NB * 256)) = S;
      const int64_t left = L - s * a.seg_len;
      const float f = left >= a.seg_len ? whole : decay(lg, (int)left);
#pragma unroll
      for (int v = 0; v < 4; ++v) S[v] = S[v] * f + x[i][v];
    }
  }
  if (a.s_out && col < d) {
#pragma unroll
    for (int v = 0; v < 4; ++v)
      if (row + v < d) a.s_out[at(v)] = S[v];
  }
}

// Sum over the partial gradients of a key head, in order: x [rows][hk][group][d] -> out
template <class T>
__global__ void __launch_bounds__(256)
    k_group_sum(const float* __restrict__ xk, const float* __restrict__ xv, int64_t B, int64_t T_, int hk, int group, int d,
                Role ok, Role ov) {
  const float* x = blockIdx.y ? xv : xk;
  const Role& o = blockIdx.y ? ov : ok;
  const int ch = d / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = id / ch;  // (b, t, head)
  if (r >= B * T_ * hk) return;
  const int col = (int)(id - r * ch) * 4;
  f32x4 s{0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < group; ++i) {
    const f32x4 y = *reinterpret_cast<const f32x4*>(x + (r * group + i) * d + col);
#pragma unroll
    for (int v = 0; v < 4; ++v) s[v] += y[v];
  }
  const int h = (int)(r % hk);
  const int64_t bt = r / hk, b = bt / T_, t = bt - b * T_;
  T* p = static_cast<T*>(const_cast<void*>(o.p)) + b * o.sb + t * o.st + h * o.sh + col;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(p) = s;
  } else {
    *reinterpret_cast<uint2*>(p) = Blk<bf16_t>::of(s);
  }
}

// One token: S' = l S + k^T v in place, o = scale q S'.  A block takes a head
// of a row, or some columns of it; a thread four columns of every RG-th row of
// the state.  Bound by the state, read and written once (200 rows of 16 heads of
// 128: 91 us, 4.6 TB/s).
template <class T, int NTHR>
__global__ void __launch_bounds__(NTHR)
    k_linattn_step(Role q, Role k, Role v, Role o, const float* __restrict__ log_decay, float* __restrict__ state,
                   const int32_t* __restrict__ slots, int64_t n_slots, int H, int d, int width, float scale) {
  __shared__ float lq[kMaxD], lk[kMaxD];
  __shared__ f32x4 part[NTHR];
  const int h = blockIdx.x % H, b = blockIdx.x / H;
  const int c0 = blockIdx.y * width, wide = d - c0 < width ? d - c0 : width;
  const int lc = wide / 4, rg = NTHR / lc;
  const int x = threadIdx.x % lc, y = threadIdx.x / lc;
  T* op = static_cast<T*>(const_cast<void*>(o.p)) + b * o.sb + (h / o.hdiv) * o.sh + c0;
  const int64_t slot = slots ? slots[b] : b;
  const bool live = slot >= 0 && slot < n_slots;
  if (live) {
    const T* qp = static_cast<const T*>(q.p) + b * q.sb + (h / q.hdiv) * q.sh;
    const T* kp = static_cast<const T*>(k.p) + b * k.sb + (h / k.hdiv) * k.sh;
    for (int i = threadIdx.x; i < d; i += NTHR) {
      lq[i] = Elt<T>::get(qp + i) * scale;
      lk[i] = Elt<T>::get(kp + i);
    }
  }
  __syncthreads();
  f32x4 s{0.f, 0.f, 0.f, 0.f};
  if (live && y < rg) {
    const float l = expf(log_decay[h]);
    const f32x4 vv = Elt<T>::load4(static_cast<const T*>(v.p) + b * v.sb + (h / v.hdiv) * v.sh + c0 + 4 * x);
    float* p = state + (slot * H + h) * (int64_t)d * d + c0 + 4 * x;
#pragma unroll 8
    for (int r = y; r < d; r += rg) {
      f32x4 w = *reinterpret_cast<const f32x4*>(p + r * d);
      const float kr = lk[r], qr = lq[r];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = fmaf(l, w[i], kr * vv[i]);
        s[i] = fmaf(qr, w[i], s[i]);
      }
      *reinterpret_cast<f32x4*>(p + r * d) = w;
    }
  }
  part[threadIdx.x] = s;
  __syncthreads();
  if (y == 0) {
    for (int i = 1; i < rg; ++i) {
      const f32x4 w = part[i * lc + x];
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += w[j];
    }
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(op + 4 * x) = s;
    } else {
      *reinterpret_cast<uint2*>(op + 4 * x) = Blk<bf16_t>::of(s);
    }
  }
}

// ---- host ---------------------------------------------------------------------------
int pad_d(int d) { return d <= 16 ? 16 : d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : 128; }

// The blocks of the walks: each takes `gr` heads, or one of `n` segments of them,
// of at least four chunks each.  As many segments as fill the chip at most once:
// 16 waves a CU fit (16 heads of 16381 tokens, d = 128: 125 to 130 us at 512 blocks,
// 136 at 256, 153 at 1024; backward of 64 x 512 tokens, 8 heads on 4, d = 64: 77
// us at 384 blocks, 118 at 768 in two segments).  Two heads a block where they
// share a key head, unless that leaves the chip short of blocks (300 tokens, 8
// heads on 4, d = 128: 32 us, 43 with two heads a block).
struct Split {
  int gr;
  int n;
  int64_t len;  // tokens of a segment, a multiple of the chunk
};
Split split_of(const hg_linattn_desc* A, int walks) {
  const int64_t heads = std::max<int64_t>(1, (int64_t)A->batch * A->heads * walks), full = 256 * (16 / (pad_d(A->d) / 16));
  const int64_t most = std::max<int64_t>(1, A->t / (4 * kChunk));
  Split p{1, 1, 0};
  if (walks > 1 && A->heads / A->kv_heads % 2 == 0 && heads / 2 * most >= full) p.gr = 2;
  const int64_t n = std::max<int64_t>(1, std::min(full / (heads / p.gr), most));
  p.len = cdiv(cdiv(std::max<int64_t>(A->t, 1), n), kChunk) * kChunk;
  p.n = (int)std::max<int64_t>(1, cdiv(A->t, p.len));
  return p;
}

// of one walk's states
int64_t seg_elems(const hg_linattn_desc* A, int walks) {
  const Split s = split_of(A, walks);
  const int64_t dp = pad_d(A->d);
  return s.n > 1 ? (int64_t)A->batch * A->heads * s.n * dp * dp : 0;
}

// `sums` of the n walks, the first ones, form their own segment sums.
template <class T, int DP, int GR>
int launch_scan(const char* name, const Walks& w, int sums, int n, int64_t B, hipStream_t s) {
  const int64_t bhs = B * w.w[0].H;
  const unsigned segs = (unsigned)w.w[0].segs;
  if (segs > 1) {
    HG_LAUNCH("linattn_sums", (k_linattn_scan<T, DP, true, 1>), dim3((unsigned)bhs, segs, sums), dim3(Shape<DP>::THREADS), 0,
              s, w);
    HG_LAUNCH("linattn_join", (k_linattn_join<DP>),
              dim3((unsigned)cdiv(bhs * (DP / 16) * (DP / 16) * 64, 256), 1, sums), dim3(256), 0, s, w, bhs);
  }
  HG_LAUNCH(name, (k_linattn_scan<T, DP, false, GR>), dim3((unsigned)(bhs / GR), segs, n), dim3(Shape<DP>::THREADS), 0, s, w);
  return HG_OK;
}

template <class T, int DP>
int scan_g(const char* name, const Walks& w, int sums, int n, int gr, int64_t B, hipStream_t s) {
  return gr == 2 ? launch_scan<T, DP, 2>(name, w, sums, n, B, s) : launch_scan<T, DP, 1>(name, w, sums, n, B, s);
}

template <class T>
int scan_d(const char* name, const Walks& w, int sums, int n, int gr, int64_t B, hipStream_t s) {
  switch (pad_d(w.w[0].d)) {
    case 16: return scan_g<T, 16>(name, w, sums, n, gr, B, s);
    case 32: return scan_g<T, 32>(name, w, sums, n, gr, B, s);
    case 64: return scan_g<T, 64>(name, w, sums, n, gr, B, s);
    case 96: return scan_g<T, 96>(name, w, sums, n, gr, B, s);
    default: return scan_g<T, 128>(name, w, sums, n, gr, B, s);
  }
}

int scan(const char* name, const hg_linattn_desc* A, const Walks& w, int sums, int n, int gr, hipStream_t s) {
  return A->dtype == HG_DTYPE_F32 ? scan_d<float>(name, w, sums, n, gr, A->batch, s)
                                  : scan_d<bf16_t>(name, w, sums, n, gr, A->batch, s);
}

int check(const hg_linattn_desc* A, const char* what) {
  if (!A) return fail(HG_ERR_ARG, "%s: null descriptor", what);
  if (A->t < 0 || A->batch < 0 || A->heads < 1 || A->kv_heads < 1 || A->d < 1)
    return fail(HG_ERR_ARG, "%s: batch=%d t=%lld heads=%d kv_heads=%d d=%d", what, A->batch, (long long)A->t, A->heads,
                A->kv_heads, A->d);
  if (A->heads % A->kv_heads) return fail(HG_ERR_ARG, "%s: %d heads on %d key heads", what, A->heads, A->kv_heads);
  if (A->dtype != HG_DTYPE_F32 && A->dtype != HG_DTYPE_BF16) return fail(HG_ERR_ARG, "%s: dtype %d", what, A->dtype);
  if (A->d % 8 || A->d > kMaxD) return fail(HG_ERR_UNSUPPORTED, "%s: d=%d is not a multiple of 8 up to %d", what, A->d, kMaxD);
  // (a grid has fewer than 2^32 threads; the end of a chunk fits 32 bits)
  if ((int64_t)A->batch * A->heads >= ((int64_t)1 << 32) / std::max(256, 4 * pad_d(A->d)) || A->t > ((int64_t)1 << 31) - 2 * kChunk ||
      A->t * A->batch > ((int64_t)1 << 36) / A->heads)
    return fail(HG_ERR_UNSUPPORTED, "%s: %d sequences of %lld tokens and %d heads are too many", what, A->batch,
                (long long)A->t, A->heads);
  return HG_OK;
}

// A strided operand: 16-byte aligned rows (null only where there are none).
int check_heads(const hg_linattn_desc* A, const char* what, const hg_heads* x, const char* name) {
  if (!x || (!x->p && A->t > 0 && A->batch > 0)) return fail(HG_ERR_ARG, "%s: null %s", what, name);
  const int64_t e = A->dtype == HG_DTYPE_F32 ? 4 : 8;
  if ((reinterpret_cast<uintptr_t>(x->p) & 15) || x->batch % e || x->token % e || x->head % e)
    return fail(HG_ERR_ARG, "%s: rows of %s are not 16-byte aligned", what, name);
  if (A->t > 1 && x->token < A->d)
    return fail(HG_ERR_ARG, "%s: tokens of %s are %lld apart, %d wide", what, name, (long long)x->token, A->d);
  if (A->t > 1 && x->token > kMaxToken)
    return fail(HG_ERR_UNSUPPORTED, "%s: tokens of %s are %lld apart", what, name, (long long)x->token);
  return HG_OK;
}

// A single token's stride is never walked: any that keeps rows apart does.
Role role(const hg_linattn_desc* A, const hg_heads* x, int hdiv) {
  return Role{x->p, x->batch, A->t > 1 ? x->token : A->d, x->head, hdiv};
}

Walk walk_of(const hg_linattn_desc* A, int walks, const float* log_decay, const int32_t* lens) {
  const Split sg = split_of(A, walks);
  Walk a{};
  a.log_decay = log_decay;
  a.lens = lens;
  a.T = A->t;
  a.seg_len = sg.len;
  a.segs = sg.n;
  a.H = A->heads;
  a.d = A->d;
  a.kv_scale = a.o_scale = 1.f;
  return a;
}

struct Bufs {
  float *seg0 = nullptr, *seg1 = nullptr;    // states of the segments: S, and in the backward R
  float *partk = nullptr, *partv = nullptr;  // gradients of k and v for each query head, or pair of them
};

template <class Mem>
Bufs take(const hg_linattn_desc* A, bool bwd, Mem& m) {
  Bufs b;
  const int walks = bwd ? 3 : 1;
  b.seg0 = m.template take<float>(seg_elems(A, walks));
  if (bwd) b.seg1 = m.template take<float>(seg_elems(A, walks));
  const int gr = split_of(A, walks).gr;
  if (bwd && A->heads / A->kv_heads > gr) {
    const int64_t n = (int64_t)A->batch * A->t * (A->heads / gr) * A->d;
    b.partk = m.template take<float>(n);
    b.partv = m.template take<float>(n);
  }
  return b;
}

int sum_groups(const hg_linattn_desc* A, const Bufs& b, const hg_heads* dk, const hg_heads* dv, hipStream_t s) {
  const int64_t rows = (int64_t)A->batch * A->t * A->kv_heads;
  if (rows == 0) return HG_OK;
  const dim3 grid((unsigned)cdiv(rows * (A->d / 4), 256), 2);
  const int group = A->heads / A->kv_heads / split_of(A, 3).gr;
  if (A->dtype == HG_DTYPE_F32) {
    HG_LAUNCH("group_sum", k_group_sum<float>, grid, dim3(256), 0, s, b.partk, b.partv, (int64_t)A->batch, A->t,
              A->kv_heads, group, A->d, role(A, dk, 1), role(A, dv, 1));
  } else {
    HG_LAUNCH("group_sum", k_group_sum<bf16_t>, grid, dim3(256), 0, s, b.partk, b.partv, (int64_t)A->batch, A->t,
              A->kv_heads, group, A->d, role(A, dk, 1), role(A, dv, 1));
  }
  return HG_OK;
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" size_t hg_linattn_fwd_workspace_size(const hg_linattn_desc* A) {
  if (check(A, "workspace size") != HG_OK) return 0;
  Sizer m;
  take(A, false, m);
  return m.used;
}

extern "C" size_t hg_linattn_bwd_workspace_size(const hg_linattn_desc* A) {
  if (check(A, "workspace size") != HG_OK) return 0;
  Sizer m;
  take(A, true, m);
  return m.used;
}

extern "C" int hg_linattn_fwd(const hg_linattn_desc* A, const hg_heads* q, const hg_heads* k, const hg_heads* v,
                              const float* log_decay, const int32_t* lens, const float* state, const hg_heads* o,
                              float* state_out, void* ws, size_t ws_bytes, void* stream) {
  const char* what = "hg_linattn_fwd";
  HG_TRY(check(A, what));
  HG_TRY(check_heads(A, what, q, "q"));
  HG_TRY(check_heads(A, what, k, "k"));
  HG_TRY(check_heads(A, what, v, "v"));
  HG_TRY(check_heads(A, what, o, "o"));
  if (A->batch == 0) return HG_OK;
  if (!log_decay) return fail(HG_ERR_ARG, "%s: null log_decay", what);
  if (A->t > 0 && (o->p == q->p || o->p == k->p || o->p == v->p)) return fail(HG_ERR_ARG, "%s: o is an input", what);
  if (state && state == state_out) return fail(HG_ERR_ARG, "%s: state_out is state", what);
  Sizer need;
  take(A, false, need);
  if (ws_bytes < need.used || (need.used && !ws))
    return fail(HG_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need.used);
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(HG_ERR_ARG, "%s: the workspace is not 16-byte aligned", what);
  Arena m(ws, ws_bytes);
  const Bufs b = take(A, false, m);
  Walks ws_{};
  Walk& a = ws_.w[0];
  a = walk_of(A, 1, log_decay, lens);
  const int group = A->heads / A->kv_heads;
  a.q = role(A, q, 1);
  a.k = role(A, k, group);
  a.v = role(A, v, group);
  a.o = role(A, o, 1);
  a.s_in = state;
  a.s_out = state_out;
  a.seg = b.seg0;
  a.o_scale = A->scale;
  return scan("linattn", A, ws_, 1, 1, 1, static_cast<hipStream_t>(stream));
}

extern "C" int hg_linattn_bwd(const hg_linattn_desc* A, const hg_heads* q, const hg_heads* k, const hg_heads* v,
                              const float* log_decay, const int32_t* lens, const float* state, const hg_heads* d_o,
                              const float* dstate_out, const hg_heads* dq, const hg_heads* dk, const hg_heads* dv,
                              float* dstate, void* ws, size_t ws_bytes, void* stream) {
  const char* what = "hg_linattn_bwd";
  hipStream_t s = static_cast<hipStream_t>(stream);
  HG_TRY(check(A, what));
  const hg_heads* all[7] = {q, k, v, d_o, dq, dk, dv};
  const char* names[7] = {"q", "k", "v", "dO", "dq", "dk", "dv"};
  for (int i = 0; i < 7; ++i) HG_TRY(check_heads(A, what, all[i], names[i]));
  if (A->batch == 0) return HG_OK;
  if (!log_decay) return fail(HG_ERR_ARG, "%s: null log_decay", what);
  for (int i = 4; i < 7 && A->t > 0; ++i)
    for (int j = 0; j < i; ++j)
      if (all[i]->p == all[j]->p) return fail(HG_ERR_ARG, "%s: %s is %s", what, names[i], names[j]);
  if (dstate && (dstate == state || dstate == dstate_out)) return fail(HG_ERR_ARG, "%s: dstate is an input", what);
  Sizer need;
  take(A, true, need);
  if (ws_bytes < need.used || (need.used && !ws))
    return fail(HG_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need.used);
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(HG_ERR_ARG, "%s: the workspace is not 16-byte aligned", what);
  Arena m(ws, ws_bytes);
  const Bufs b = take(A, true, m);
  const int group = A->heads / A->kv_heads, gr = split_of(A, 3).gr;
  const int64_t H = A->heads / gr, d = A->d;  // of the partial gradients
  Walks w{};
  Walk &wq = w.w[0], &wv = w.w[1], &wk = w.w[2];
  wq = wv = walk_of(A, 3, log_decay, lens);
  // dq: its state is the transpose of the forward's
  wq.q = role(A, d_o, 1);
  wq.k = role(A, v, group);
  wq.v = role(A, k, group);
  wq.o = role(A, dq, 1);
  wq.s_in = state;
  wq.s_trans = 1;
  wq.seg = b.seg0;
  wq.o_scale = A->scale;
  // dv: from the last token, for each query head
  wv.reverse = 1;
  wv.kv_scale = A->scale;
  wv.q = role(A, k, group);
  wv.k = role(A, q, 1);
  wv.v = role(A, d_o, 1);
  wv.o = group > gr ? Role{b.partv, A->t * H * d, H * d, d, gr} : role(A, dv, group);
  wv.f32_out = group > gr;
  wv.sum_o = 1;
  wv.s_in = dstate_out;
  wv.s_out = dstate;
  wv.seg = b.seg1;
  // dk: its state is the transpose of dv's
  wk = wv;
  wk.q = role(A, v, group);
  wk.k = role(A, d_o, 1);
  wk.v = role(A, q, 1);
  wk.o = group > gr ? Role{b.partk, A->t * H * d, H * d, d, gr} : role(A, dk, group);
  wk.s_trans = 1;
  wk.seg_trans = 1;
  wk.s_out = nullptr;
  HG_TRY(scan("linattn_bwd", A, w, 2, 3, gr, s));
  if (group > gr) HG_TRY(sum_groups(A, b, dk, dv, s));
  return HG_OK;
}

extern "C" int hg_linattn_step(const hg_linattn_desc* A, const hg_heads* q, const hg_heads* k, const hg_heads* v,
                               const float* log_decay, float* state, const int32_t* slots, int64_t n_slots,
                               const hg_heads* o, void* stream) {
  const char* what = "hg_linattn_step";
  hipStream_t s = static_cast<hipStream_t>(stream);
  HG_TRY(check(A, what));
  if (A->t != 1) return fail(HG_ERR_ARG, "%s: t=%lld, one token a row", what, (long long)A->t);
  HG_TRY(check_heads(A, what, q, "q"));
  HG_TRY(check_heads(A, what, k, "k"));
  HG_TRY(check_heads(A, what, v, "v"));
  HG_TRY(check_heads(A, what, o, "o"));
  if (n_slots < 0 || (!slots && n_slots < A->batch))
    return fail(HG_ERR_ARG, "%s: %lld states for %d rows", what, (long long)n_slots, A->batch);
  if (A->batch == 0) return HG_OK;
  if (!log_decay || (!state && n_slots > 0)) return fail(HG_ERR_ARG, "%s: null pointer", what);
  if (reinterpret_cast<uintptr_t>(state) & 15) return fail(HG_ERR_ARG, "%s: the states are not 16-byte aligned", what);
  // (blocks of the same row, and of heads that share k and v, read their inputs while another writes o)
  if (o->p == q->p || o->p == k->p || o->p == v->p) return fail(HG_ERR_ARG, "%s: o is an input", what);
  // whole heads while there are two blocks per CU of them, else columns of a
  // head, at least 16 (64 bytes of a row of the state)
  const int64_t heads = (int64_t)A->batch * A->heads;
  int width = A->d;
  while (width > 16 && heads * cdiv(A->d, width) < 512) width = std::max(16, (int)cdiv(width / 2, 8) * 8);
  const int group = A->heads / A->kv_heads;
  const dim3 grid((unsigned)heads, (unsigned)cdiv(A->d, width));
#define HG_STEP(T_, N_)                                                                                              \
  HG_LAUNCH("linattn_step", (k_linattn_step<T_, N_>), grid, dim3(N_), 0, s, role(A, q, 1), role(A, k, group), role(A, v, group), \
            role(A, o, 1), log_decay, state, slots, n_slots, A->heads, A->d, width, A->scale)
  const bool small = A->d <= 32;
  if (A->dtype == HG_DTYPE_F32) {
    if (small) {
      HG_STEP(float, 64);
    } else {
      HG_STEP(float, 256);
    }
  } else if (small) {
    HG_STEP(bf16_t, 64);
  } else {
    HG_STEP(bf16_t, 256);
  }
#undef HG_STEP
  return HG_OK;
}
