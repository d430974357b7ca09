// What the kernels over pages of 8-bit codes share: where a slot lies, codes and scales, and the rotary embedding of rows.
#pragma once
#include "ig_internal.h"

struct PageRefs {
  const int32_t *table;               // [B][stride]
  char *K, *V;                        // [n_pages][H][page][d]
  float *K_scale, *V_scale;           // [n_pages][H]
  unsigned n_pages, page_bytes;       // of all heads
  int stride, shift, H;               // a page has 1 << shift slots
};
static inline PageRefs ig_page_refs(const ig_desc *d, const ig_pages *p) {
  PageRefs r;
  r.table = p->table, r.K = static_cast<char *>(p->K), r.V = static_cast<char *>(p->V), r.K_scale = p->K_scale, r.V_scale = p->V_scale;
  r.n_pages = (unsigned)p->n_pages, r.page_bytes = (unsigned)(d->H * p->page_size * d->d);
  r.stride = p->table_stride, r.shift = __builtin_ctz(p->page_size), r.H = d->H;
  return r;
}
// an entry of the table as a page that may be read
__device__ __forceinline__ unsigned page_read(const PageRefs &p, int entry) { return min((unsigned)max(entry, 0), p.n_pages - 1); }

// Scales are powers of two, so that rounding a value by one is exact, a page's codes can be rounded again to a larger one
// with errors that halve every time, and a scale is its exponent.
constexpr int SCALE_LEAST = -80, SCALE_MOST = 122;
template <int MOST = SCALE_MOST> __device__ __forceinline__ int scale_exponent(float s) {
  return min(max((int)(__float_as_uint(s) >> 23 & 255) - 127, SCALE_LEAST), MOST);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }      // -126 <= e <= 127
// The least exponent e with top <= most * 2^e: most is 127 = 1.984375 * 2^6, or 448 = 1.75 * 2^8.
template <bool E4M3> __device__ __forceinline__ int exponent_for(float top) {
  const unsigned bits = __float_as_uint(top);
  const int e = (int)(bits >> 23 & 255) - 127 - (E4M3 ? 8 : 6) + ((bits & 0x7fffffu) > (E4M3 ? 0x600000u : 0x7e0000u));
  return min(max(e, SCALE_LEAST), SCALE_MOST);
}

// four values, multiples of a scale already, as four codes: the nearest, ties to the even one
template <bool E4M3> __device__ __forceinline__ unsigned encode4(float a, float b, float c, float d) {
  if constexpr (E4M3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
  } else {
    const unsigned x = (unsigned)(int)rintf(a), y = (unsigned)(int)rintf(b), z = (unsigned)(int)rintf(c), w = (unsigned)(int)rintf(d);
    const unsigned lo = __builtin_amdgcn_perm(y, x, 0x0c0c0400u), hi = __builtin_amdgcn_perm(w, z, 0x04000c0cu);
    return lo | hi;
  }
}
template <bool E4M3> __device__ __forceinline__ floatx4 decode4(unsigned v) {
  if constexpr (E4M3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, true);
    return floatx4{lo[0], lo[1], hi[0], hi[1]};
  } else {
    return floatx4{(float)(int8_t)v, (float)(int8_t)(v >> 8), (float)(int8_t)(v >> 16), (float)(int8_t)(v >> 24)};
  }
}

// ---- rotary embedding ----------------------------------------------------------------------------------------------
// A thread takes units of 16 channels of a row, eight pairs a_e, b_e.  The first dims/2 pairs of a row's are rotated, pair c
// by freq[c]; channels past dims are pairs that stay.  Where pairs are (c, c + dims/2) with dims a multiple of 16, and where
// they are next to each other, a unit is two runs of eight channels; else its channels are taken one by one.  No two units share
// a channel, so rows may be rotated in place.
enum Turn { TURN_NONE, TURN_HALVES, TURN_ADJACENT, TURN_ANY };
struct RotaryRefs {
  const double *freq;
  float magnitude, sign;              // -1: the transpose
  int dims, kind;
};
static inline RotaryRefs ig_rotary_refs(const ig_rotary *r, int inverse) {
  if (!r) return RotaryRefs{nullptr, 1.f, 1.f, 0, TURN_NONE};
  return RotaryRefs{r->freq, r->magnitude, inverse ? -1.f : 1.f, r->dims, r->interleaved ? TURN_ADJACENT : (r->dims % 16 ? TURN_ANY : TURN_HALVES)};
}
struct Runs {
  int first, second;
};
template <int KIND> __device__ __forceinline__ Runs runs_of(int s, int dims) {
  const bool halves = KIND == TURN_HALVES && 16 * s < dims;
  return Runs{halves ? 8 * s : 16 * s, halves ? 8 * s + dims / 2 : 16 * s + 8};
}
// TURN_ANY: channel x (0: a, 1: b) of pair c
__device__ __forceinline__ int any_channel(int c, int x, int dims) {
  return 2 * c < dims ? c + (x ? dims / 2 : 0) : 2 * c + x;
}
// Cosine and sine of pos * freq: the product and the reduction to a quarter turn in double (a float32 angle of a far position
// has no phase left), the Taylor polynomials to x^13 and x^12 in float32 on [-pi/4, pi/4] (truncation below 2^-40).
__device__ __forceinline__ float2 turn_of(int pos, double freq, const RotaryRefs &r) {
  const double angle = (double)pos * freq, k = rint(angle * 0.63661977236758134308);      // 2 / pi
  const float x = (float)fma(-k, 6.12323399573676603587e-17, fma(-k, 1.57079632679489655800e+00, angle)), x2 = x * x;
  float c = 1.f, s = 1.f;
#pragma unroll
  for (int n = 6; n >= 1; --n) {
    c = fmaf(-x2 * (1.f / (float)((2 * n - 1) * (2 * n))), c, 1.f);
    s = fmaf(-x2 * (1.f / (float)((2 * n) * (2 * n + 1))), s, 1.f);
  }
  s *= x;
  const int q = (int)(long long)k & 3;
  const float cs = q & 1 ? s : c, sn = q & 1 ? c : s;
  return make_float2((q == 1 || q == 2 ? -cs : cs) * r.magnitude, (q >= 2 ? -sn : sn) * r.magnitude * r.sign);
}
// the eight pairs of unit s (a pair past the last one: any)
__device__ __forceinline__ void turns_of(int s, int pos, const RotaryRefs &r, float2 (&turn)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = 8 * s + e;
    turn[e] = turn_of(pos, r.freq[min(c, r.dims / 2 - 1)], r);
    // (two at a time: all at once they take more registers than there are)
    if (e % 2) asm volatile("" : "+v"(turn[e - 1].x), "+v"(turn[e - 1].y), "+v"(turn[e].x), "+v"(turn[e].y));
  }
}
// eight values of a row
template <typename T> struct Run8;
template <> struct Run8<half_t> {
  uint4 v;
  __device__ __forceinline__ void load(const half_t *p) { v = *reinterpret_cast<const uint4 *>(p); }
  __device__ __forceinline__ void set(int e, half_t x) {
    half8 h = __builtin_bit_cast(half8, v);
    h[e] = x;
    v = __builtin_bit_cast(uint4, h);
  }
  __device__ __forceinline__ void get(float *x) const {
    const half8 h = __builtin_bit_cast(half8, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
  }
  static __device__ __forceinline__ void store(half_t *p, const float *x) {
    half8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (half_t)x[e];
    *reinterpret_cast<uint4 *>(p) = __builtin_bit_cast(uint4, h);
  }
};
template <> struct Run8<float> {
  floatx4 v[2];
  __device__ __forceinline__ void load(const float *p) {
    v[0] = reinterpret_cast<const floatx4 *>(p)[0], v[1] = reinterpret_cast<const floatx4 *>(p)[1];
  }
  __device__ __forceinline__ void set(int e, float x) { v[e / 4][e % 4] = x; }
  __device__ __forceinline__ void get(float *x) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e / 4][e % 4];
  }
  static __device__ __forceinline__ void store(float *p, const float *x) {
    reinterpret_cast<floatx4 *>(p)[0] = floatx4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<floatx4 *>(p)[1] = floatx4{x[4], x[5], x[6], x[7]};
  }
};

// a unit's values: x[0 .. 7] the first run, x[8 .. 15] the second (channels one by one: the pairs' a, the pairs' b)
template <typename T, int KIND> struct Unit {
  Run8<T> lo, hi;
  static __device__ __forceinline__ bool one_by_one(int dims) { return KIND == TURN_ANY && dims > 0; }
  __device__ __forceinline__ void load(const T *row, int s, int dims) {
    if (one_by_one(dims)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) lo.set(e, row[any_channel(8 * s + e, 0, dims)]), hi.set(e, row[any_channel(8 * s + e, 1, dims)]);
      return;
    }
    const Runs c = runs_of<KIND>(s, dims);
    lo.load(row + c.first);
    hi.load(row + c.second);
  }
  __device__ __forceinline__ void get(float (&x)[16]) const {
    lo.get(x);
    hi.get(x + 8);
  }
  static __device__ __forceinline__ void store(T *row, int s, int dims, const float (&x)[16]) {
    if (one_by_one(dims)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) row[any_channel(8 * s + e, 0, dims)] = (T)x[e], row[any_channel(8 * s + e, 1, dims)] = (T)x[8 + e];
      return;
    }
    const Runs c = runs_of<KIND>(s, dims);
    Run8<T>::store(row + c.first, x);
    Run8<T>::store(row + c.second, x + 8);
  }
};
// (channels that stay are not multiplied: an infinity there would make a NaN of its neighbour)
template <int KIND> __device__ __forceinline__ void rotate_unit(float (&x)[16], int s, int dims, const float2 (&turn)[8]) {
  if (KIND == TURN_NONE || 16 * s >= dims) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    constexpr int A = KIND == TURN_ADJACENT ? 2 : 1, B = KIND == TURN_ADJACENT ? 1 : 8;
    const float a = x[A * e], b = x[A * e + B], y = fmaf(a, turn[e].x, -b * turn[e].y), z = fmaf(b, turn[e].x, a * turn[e].y);
    const bool turns = KIND == TURN_HALVES || 2 * (8 * s + e) < dims;
    x[A * e] = turns ? y : a, x[A * e + B] = turns ? z : b;
  }
}
