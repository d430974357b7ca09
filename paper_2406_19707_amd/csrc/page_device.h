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
  r.n_pages = (unsigned)p->n_pages, r.page_bytes = (unsigned)d->H * (unsigned)p->page_size * (unsigned)d->d;      // (at most 2^31)
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
// by freq[c]; channels past dims are pairs that stay.  Pairs next to each other make a unit of two runs of eight channels.  Pairs
// (c, c + dims/2) are taken in runs of as many as divide dims/2, eight where they can be: a run of a's and a run of b's.  No two
// units share a channel, so rows may be rotated in place.
enum Turn { TURN_NONE, TURN_ADJACENT, TURN_HALVES, TURN_HALVES_4, TURN_HALVES_2, TURN_HALVES_1 };
constexpr int run_of(int kind) { return kind == TURN_HALVES_4 ? 4 : kind == TURN_HALVES_2 ? 2 : kind == TURN_HALVES_1 ? 1 : 8; }
struct RotaryRefs {
  const double *freq;
  float magnitude, sign;              // -1: the transpose
  int dims, kind;
};
static inline RotaryRefs ig_rotary_refs(const ig_rotary *r, int inverse) {
  if (!r) return RotaryRefs{nullptr, 1.f, 1.f, 0, TURN_NONE};
  const int half = r->dims / 2, halves = half % 8 == 0 ? TURN_HALVES : half % 4 == 0 ? TURN_HALVES_4 : half % 2 == 0 ? TURN_HALVES_2 : TURN_HALVES_1;
  return RotaryRefs{r->freq, r->magnitude, inverse ? -1.f : 1.f, r->dims, r->interleaved ? TURN_ADJACENT : halves};
}
// where the a's and the b's of the run of pairs from pair c on begin
struct Runs {
  int first, second;
};
template <int KIND> __device__ __forceinline__ Runs runs_of(int c, int dims) {
  const bool halves = KIND >= TURN_HALVES && 2 * c < dims;
  return Runs{halves ? c : 2 * c, halves ? c + dims / 2 : 2 * c + run_of(KIND)};
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
// N values of a row, up to 16 bytes a load
template <typename T, int N> struct RunOf {
  static constexpr int PER = N * (int)sizeof(T) <= 16 ? N : 16 / (int)sizeof(T);
  typedef T vec __attribute__((ext_vector_type(PER)));
  vec v[N / PER];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < N / PER; ++i) v[i] = reinterpret_cast<const vec *>(p)[i];
  }
  __device__ __forceinline__ void get(float *x) const {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (float)v[e / PER][e % PER];
  }
  static __device__ __forceinline__ void store(T *p, const float *x) {
#pragma unroll
    for (int i = 0; i < N / PER; ++i) {
      vec y;
#pragma unroll
      for (int e = 0; e < PER; ++e) y[e] = (T)x[i * PER + e];
      reinterpret_cast<vec *>(p)[i] = y;
    }
  }
};
// a unit's values: x[0 .. 7] the a's (of pairs next to each other: the first run), x[8 .. 15] the b's (the second)
template <typename T, int KIND> struct Unit {
  static constexpr int G = run_of(KIND);
  RunOf<T, G> lo[8 / G], hi[8 / G];
  __device__ __forceinline__ void load(const T *row, int s, int dims) {
#pragma unroll
    for (int j = 0; j < 8 / G; ++j) {
      const Runs c = runs_of<KIND>(8 * s + G * j, dims);
      lo[j].load(row + c.first);
      hi[j].load(row + c.second);
    }
  }
  __device__ __forceinline__ void get(float (&x)[16]) const {
#pragma unroll
    for (int j = 0; j < 8 / G; ++j) {
      lo[j].get(x + G * j);
      hi[j].get(x + 8 + G * j);
    }
  }
  static __device__ __forceinline__ void store(T *row, int s, int dims, const float (&x)[16]) {
#pragma unroll
    for (int j = 0; j < 8 / G; ++j) {
      const Runs c = runs_of<KIND>(8 * s + G * j, dims);
      RunOf<T, G>::store(row + c.first, x + G * j);
      RunOf<T, G>::store(row + c.second, x + 8 + G * j);
    }
  }
  // the same of codes, four a word: c[0], c[1] those of x[0 .. 7], c[2], c[3] of x[8 .. 15]
  static __device__ __forceinline__ void store_codes(char *row, int s, int dims, const unsigned (&c)[4]) {
#pragma unroll
    for (int j = 0; j < 8 / G; ++j) {
      const Runs at = runs_of<KIND>(8 * s + G * j, dims);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        char *to = row + (b ? at.second : at.first);
        if constexpr (G == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(c[2 * b], c[2 * b + 1]);
        else if constexpr (G == 4) *reinterpret_cast<unsigned *>(to) = c[2 * b + j];
        else if constexpr (G == 2) *reinterpret_cast<unsigned short *>(to) = (unsigned short)(c[2 * b + j / 2] >> j % 2 * 16);
        else *to = (char)(c[2 * b + j / 4] >> j % 4 * 8);
      }
    }
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
