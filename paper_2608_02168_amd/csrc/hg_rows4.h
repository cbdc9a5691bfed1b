// Rows of channels at any alignment of their own values, for the operators that
// only pass over them once (recurrence, group norm): a sequence's token and
// channel lie at p[b * sb + t * st + c], and a thread takes V adjacent channels
// with one load (the hardware takes any address that is a multiple of the
// value's size).
#pragma once

#include <algorithm>

#include "hg_mfma.h"

namespace hg {

struct Rows {
  void* p;
  int64_t sb, st;
};

// V adjacent values, as loaded (raw), one by one (get), and written (put).
template <class T, int V>
struct Vec;
template <int V>
struct Vec<float, V> {
  typedef float raw __attribute__((ext_vector_type(V), aligned(4)));
  __device__ static __forceinline__ raw load(const float* p) { return *reinterpret_cast<const raw*>(p); }
  __device__ static __forceinline__ float get(const raw& x, int j) { return x[j]; }
  __device__ static __forceinline__ void put(float* p, const float (&v)[V]) {
    raw x;
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = v[j];
    *reinterpret_cast<raw*>(p) = x;
  }
};
template <>
struct Vec<float, 1> {
  typedef float raw;
  __device__ static __forceinline__ raw load(const float* p) { return *p; }
  __device__ static __forceinline__ float get(const raw& x, int) { return x; }
  __device__ static __forceinline__ void put(float* p, const float (&v)[1]) { *p = v[0]; }
};
template <int V>
struct Vec<bf16_t, V> {
  typedef uint32_t raw __attribute__((ext_vector_type(V / 2), aligned(2)));
  __device__ static __forceinline__ raw load(const bf16_t* p) { return *reinterpret_cast<const raw*>(p); }
  __device__ static __forceinline__ float get(const raw& x, int j) {
    return __uint_as_float(j & 1 ? x[j >> 1] & 0xFFFF0000u : x[j >> 1] << 16);
  }
  __device__ static __forceinline__ void put(bf16_t* p, const float (&v)[V]) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    raw x;
#pragma unroll
    for (int j = 0; j < V / 2; ++j)
      x[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{v[2 * j], v[2 * j + 1]}), b2));
    *reinterpret_cast<raw*>(p) = x;
  }
};
template <>
struct Vec<bf16_t, 1> {
  typedef uint16_t raw;
  __device__ static __forceinline__ raw load(const bf16_t* p) { return *p; }
  __device__ static __forceinline__ float get(const raw& x, int) { return bf2f(x); }
  __device__ static __forceinline__ void put(bf16_t* p, const float (&v)[1]) { *p = f2bf(v[0]); }
};

// ---- host: checks that the operators over such rows share ----------------------
constexpr int64_t kMaxRowStride = (int64_t)1 << 40;

// Rows [batch, t, width] of dtype (null only where there are none); out: rows apart.
inline int check_rows(const char* what, const hg_heads* x, const char* name, bool out, int64_t batch, int64_t t, int32_t width,
                      int32_t dtype) {
  if (!x || (!x->p && t > 0 && batch > 0)) return fail(HG_ERR_ARG, "%s: null %s", what, name);
  const uintptr_t e = dtype == HG_DTYPE_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(x->p) % e) return fail(HG_ERR_ARG, "%s: %s is not aligned to its values", what, name);
  if (x->batch < 0 || x->token < 0 || x->batch > kMaxRowStride || x->token > kMaxRowStride)
    return fail(HG_ERR_ARG, "%s: strides %lld, %lld of %s", what, (long long)x->batch, (long long)x->token, name);
  // sequence by sequence, or token by token
  const bool apart = (t <= 1 || x->token >= width) && (batch <= 1 || x->batch >= width) &&
                     (t <= 1 || batch <= 1 || x->batch >= (t - 1) * x->token + width || x->token >= (batch - 1) * x->batch + width);
  if (out && !apart)
    return fail(HG_ERR_ARG, "%s: rows of %s overlap (strides %lld, %lld, %d wide)", what, name, (long long)x->batch,
                (long long)x->token, width);
  return HG_OK;
}

// Whether an output's rows o may share an address with the rows x: not if they lie in
// different stretches of memory; with the same strides (views of one buffer) exactly if
// some two rows are less than a row's width apart.
inline bool rows_meet(const hg_heads* o, const hg_heads* x, int64_t batch, int64_t t, int32_t width, int32_t dtype) {
  if (t < 1 || batch < 1) return false;
  const int64_t e = dtype == HG_DTYPE_F32 ? 4 : 2;
  const auto bytes = [&](const hg_heads* h) { return ((batch - 1) * h->batch + (t - 1) * h->token + width) * e; };
  const intptr_t po = reinterpret_cast<intptr_t>(o->p), px = reinterpret_cast<intptr_t>(x->p);
  if (po + bytes(o) <= px || px + bytes(x) <= po) return false;
  if ((t > 1 && o->token != x->token) || (batch > 1 && o->batch != x->batch)) return true;
  if ((px - po) % e) return true;
  // Rows (b, t) of o and (b', t') of x start d - k2 outer - k1 inner values apart, k1 and k2 any
  // differences of their indexes.  An outer step is longer than all inner ones with a row
  // (check_rows), so only the two k2 next to d matter, and for each the two k1 next to what is left.
  struct Step {
    int64_t stride, most;
  } inner{t > 1 ? o->token : 1, t - 1}, outer{batch > 1 ? o->batch : 1, batch - 1};
  if (inner.stride > outer.stride) std::swap(inner, outer);
  const auto near = [](int64_t d, const Step& s, int up) {
    const int64_t k = d / s.stride - (d % s.stride < 0) + up;
    return d - std::min(std::max(k, -s.most), s.most) * s.stride;
  };
  const int64_t d = (px - po) / e;
  for (int a = 0; a < 2; ++a)
    for (int b = 0; b < 2; ++b) {
      const int64_t apart = near(near(d, outer, a), inner, b);
      if (apart > -width && apart < width) return true;
    }
  return false;
}

// Whether two stretches of memory share an address (not if either is null or empty).
inline bool ranges_meet(const void* p, size_t a, const void* q, size_t b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
  return p && q && a && b && x < y + b && y < x + a;
}

inline Rows rows_of(const hg_heads* x) { return Rows{x->p, x->batch, x->token}; }

inline int check_workspace(const char* what, const void* ws, size_t ws_bytes, size_t need) {
  if (ws_bytes < need || (need && !ws))
    return fail(HG_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need);
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(HG_ERR_ARG, "%s: the workspace is not 16-byte aligned", what);
  return HG_OK;
}

}  // namespace hg
