// Attention over pages of 8-bit codes with a scale for each page and head: softmax(q K^T) V of a prompt, a chunk of one or a
// single token, with K = 2^ek codes and V = 2^ev codes.
#include <type_traits>

#include "cache_device.h"
#include "page_device.h"

namespace {

// ---- codes as operands -----------------------------------------------------------------------------------------------
// Every code is a half exactly, so products with codes are those of half precision: eight codes as an operand.
// An int8 code with its sign bit flipped is c + 128, and 0x6400 with that as its low byte the half 1024 + c + 128.
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
template <bool E4M3> __device__ __forceinline__ uint2 halves_of(unsigned codes) {
  if constexpr (E4M3) {
    return make_uint2(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.f, false)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.f, true)));
  } else {
    const unsigned u = codes ^ 0x80808080u, x = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u), y = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
    const half2v off = {(half_t)1152.f, (half_t)1152.f};
    return make_uint2(__builtin_bit_cast(unsigned, __builtin_bit_cast(half2v, x) - off), __builtin_bit_cast(unsigned, __builtin_bit_cast(half2v, y) - off));
  }
}
template <bool E4M3> __device__ __forceinline__ half8 operand_of(unsigned lo, unsigned hi) {
  const uint2 a = halves_of<E4M3>(lo), b = halves_of<E4M3>(hi);
  return __builtin_bit_cast(half8, make_uint4(a.x, a.y, b.x, b.y));
}
// the words of four rows as the words of four columns: byte r of word c is byte c of row r
__device__ __forceinline__ void transpose4(const unsigned (&r)[4], unsigned (&c)[4]) {
  const unsigned a = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), b = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u);
  const unsigned x = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u), y = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
  c[0] = __builtin_amdgcn_perm(b, a, 0x05040100u), c[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  c[2] = __builtin_amdgcn_perm(y, x, 0x05040100u), c[3] = __builtin_amdgcn_perm(y, x, 0x07060302u);
}

// W words as load_words loads them, past the caches where they are read ONCE.  (V's: its loads are whole rows.  16 x 32 heads of 4096
// 95 -> 86 us, 16 x 8 ragged of 32768 131 -> 121, float32 16 x 32 of 4096 99 -> 90, d = 256 100 -> 91, d = 64 as before.  K's too: 87
// and 127, as a load is half of its rows' lines.)
template <int W, bool ONCE> __device__ __forceinline__ void load_codes_of(const char *from, unsigned (&to)[W]) {
  if constexpr (!ONCE) {
    load_words<W>(from, to);
  } else {
    typedef unsigned vec __attribute__((ext_vector_type(W < 4 ? W : 4)));
    constexpr int PER = W < 4 ? W : 4;
#pragma unroll
    for (int i = 0; i < W / PER; ++i) {
      const vec x = __builtin_nontemporal_load(reinterpret_cast<const vec *>(from) + i);
#pragma unroll
      for (int e = 0; e < PER; ++e) to[i * PER + e] = x[e];
    }
  }
}

// K's largest scale: with half-precision queries less, so that its product with the logits' scale stays finite
template <bool F32> constexpr int k_scale_most() { return F32 ? SCALE_MOST : 100; }
// The factor of the logits, from K's scale and the queries' or the logits' own: above zero, so that a masked slot's -infinity stays one,
// and finite, so that a product of zero stays zero.  (Products of codes and queries are below 2^34: at 2^-126 a logit is zero either way.)
__device__ __forceinline__ float factor_of(float k, float own) { return __builtin_amdgcn_fmed3f(k * own, 0x1p-126f, 0x1.fffffep127f); }

// Float32: a lane's sum is worked out without its page's scale of V where its largest weight times scale is below 2^FAR.  With ev >=
// SCALE_LEAST such a lane's logits are 10 or more below the reference, which is at most SCALE_MOST above the largest logit: what
// counts of 2^(logit - reference) lies between about 2^-(SCALE_MOST + 30) and 2^-10, and 2^FAR_LIFT times that is in range.  (In half precision a weight that is lost
// so belongs to a row with a weight times scale of 2^46 of its largest weight and more: infinite where that one's code is not zero, and
// where it is, the others are below what weights as halves keep.)
constexpr float FAR = -90.f;
constexpr int FAR_LIFT = 64;

// a float as two halves: x - hi - lo is at most 2^-22 |x|, or 2^-25
struct Halves {
  half_t hi, lo;
};
__device__ __forceinline__ Halves split(float x) {
  const half_t hi = (half_t)x;
  return Halves{hi, (half_t)(x - (float)hi)};
}

// ---- few query rows, many cached rows ----------------------------------------------------------------------------------
// As over a pool of rows (attend_stream): S^T = K Q^T and O^T = V^T P^T on 16x16x32 products, a query row a column, tiles of 32
// slots dealt to the four waves of a workgroup, each with its own running reference, sums and outputs, nothing of K or V
// through LDS.  Lane (i, g) = (lane % 16, lane / 16):
//  - row i of the 16-row block m of S^T is the tile's slot 8 (i/4) + 4 m + i%4; a lane holds 16 bytes of every 64 of it (d = 32:
//    8 of 32), so that a load is whole sectors of 16 rows, and the queries in the same order;
//  - it supplies the weights of slots 8g .. 8g+7 and holds d/16 channels of V's rows there, whose bytes are transposed four
//    by four.  Those eight slots lie in one page: its scales are the lane's.
// K's scale goes into the factor of the logits.  V's scale 2^ev goes into the exponent of the weights, which are
// exp2(l + ev - ref) with ref the largest l + ev (or LIFT less): so no page's scale takes them out of half precision's range, and
// sums take them times 2^-ev, or without ev where a page of small values beside one of large ones would take all of a lane's
// weights below the smallest float (FAR): outputs do without them, but not the sum.  Float32 queries and weights are two halves each, and their products two.
// Bound by memory: one token of 16 x 32 heads over 4096 slots, d = 128, 84 us = 6.4 TB/s (a plain read reaches 6.3; the same over halves
// 177), of 16 x 8 x 4 ragged heads over 32768 116 us = 6.0 among other calls (121 on a GPU that was idle before); float32 16 x 32 over 4096 90 us.  V is asked for with K, a turn ahead:
// asked for after its own turn's products, 8 x 32 heads of 2048 took 32 us instead of 31.
template <int D, int NT, bool E4M3, bool F32, bool ONCE>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void page_stream(StreamArgs a, PageRefs p) {
  typedef typename std::conditional<F32, float, half_t>::type T;
  constexpr int TT = 32, CJ = D / 16, RB = 16 * NT, KS = D / 32, PARTS = F32 ? 2 : 1;
  constexpr int KB = D < 64 ? 8 : 16, KW = D / 16;        // bytes of a load of K; words of a lane's part of a row
  constexpr int VB = CJ, VW = (VB + 3) / 4;               // bytes and words of a lane's part of a V row
  constexpr float LIFT = 14.f;
  constexpr int LDB = D + 4;
  __shared__ __attribute__((aligned(16))) float boxes[4][RB * LDB];
  __shared__ float box_m[4][RB], box_l[4][RB];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  int work = xcd_order(blockIdx.x, a.per_xcd);
  if (work >= a.total) return;
  const int h = a.by_pair.div(work);
  work -= h * (int)a.by_pair.d;
  const int number = a.by_units.div(work), rb = a.nrb - 1 - a.by_units.mod(work);
  const Span span = span_of<false>(a, number);
  if (span.b < 0) return;
  const int b = span.b, kv = span.kv, nq = span.nq;

  const int first_row = rb * RB, last_row = min(min(a.R, nq * (int)a.by_group.d), first_row + RB) - 1;
  const bool rows_here = last_row >= first_row;
  const int lim_min = rows_here ? row_limit<false>(a, first_row, kv, nq) : 0x7fffffff;
  const int cached = rows_here ? row_limit<false>(a, last_row, kv, nq) : 0, tiles = (cached + TT - 1) / TT;
  const int per = (tiles + span.slices - 1) / span.slices;
  const int t_begin = min(tiles, span.slice * per), t_end = min(tiles, t_begin + per);

  const int32_t *table = p.table + (long)b * p.stride;
  const unsigned in_page = (1u << p.shift) - 1;
  const char *Kh = p.K + ((unsigned long)h << p.shift) * D, *Vh = p.V + ((unsigned long)h << p.shift) * D;
  // (slots past the last one that a row sees are read from that one)
  const int last = cached - 1;
  auto page_at = [&](int tile) __attribute__((always_inline)) { return page_read(p, table[min(tile * TT + 8 * g, last) >> p.shift]); };
  unsigned k[2][KW], v[2][8][VW];                         // (of V this tile's and the next one's)
  float ks = 1.f, vs[2] = {1.f, 1.f};
  auto load_k = [&](int tile, unsigned page) __attribute__((always_inline)) {
    const unsigned k_page = (unsigned)__shfl((int)page, (i >> 2) * 16, 64);
    const char *base = Kh + (unsigned long)k_page * p.page_bytes + g * KB;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int c = 0; c < D / (4 * KB); ++c)
        load_words<KB / 4>(base + (min(tile * TT + 8 * (i >> 2) + 4 * m + (i & 3), last) & in_page) * D + c * 4 * KB,
                           reinterpret_cast<unsigned (&)[KB / 4]>(k[m][c * (KB / 4)]));
    ks = p.K_scale[(unsigned long)page * p.H + h];
  };
  auto load_v = [&](int tile, unsigned page, unsigned (&v)[8][VW], float &vs) __attribute__((always_inline)) {
    const char *base = Vh + (unsigned long)page * p.page_bytes + VB * i;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const char *from = base + (min(tile * TT + 8 * g + u, last) & in_page) * D;
      if constexpr (VB == 2) v[u][0] = *reinterpret_cast<const unsigned short *>(from);
      else load_codes_of<VW, ONCE>(from, v[u]);
    }
    vs = p.V_scale[(unsigned long)page * p.H + h];
  };

  int tile = t_begin + w;
  unsigned page = 0, page_next = 0;
  if (tile < t_end) {
    page = page_at(tile);
    page_next = page_at(tile + 4);
  }
  int lim[NT];
  float q_scale[NT];                                      // of a row's logits, but for K's scale
  half8 qf[NT][PARTS][KS];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = rb * RB + n * 16 + i, iq = a.by_group.div(row), gq = row - iq * (int)a.by_group.d;
    lim[n] = row <= last_row ? row_limit<false>(a, row, kv, nq) : 0x7fffffff;
    const T *src = static_cast<const T *>(a.q) + (((long)b * a.n_q + min(iq, a.n_q - 1)) * a.Hq + h * (int)a.by_group.d + gq) * D;
    // (the eight channels of product c of this lane)
    auto channel = [&](int c) { return KB == 8 ? 8 * g : c / 2 * 64 + g * 16 + c % 2 * 8; };
    q_scale[n] = a.c;
    if constexpr (!F32) {
#pragma unroll
      for (int c = 0; c < KS; ++c) qf[n][0][c] = __builtin_bit_cast(half8, flip_sign<half_t>(*reinterpret_cast<const uint4 *>(src + channel(c)), a.flip));
    } else {
      // a row's largest value comes to 2^13 .. 2^14, so that what the two halves leave is 2^-38 of it at most
      float x[KS * 8], top = 0.f;
#pragma unroll
      for (int c = 0; c < KS * 2; ++c) {
        const floatx4 f = __builtin_bit_cast(floatx4, flip_sign<float>(reinterpret_cast<const uint4 *>(src + channel(c / 2))[c % 2], a.flip));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[c * 4 + e] = f[e], top = fmaxf(top, fabsf(f[e]));
      }
      const int e = min(max((int)(__float_as_uint(column_max(top)) >> 23), 20), 254) - 127;
      const float by = exp2_int(13 - e);
      q_scale[n] = exp2_int(e - 13) * a.c;
#pragma unroll
      for (int c = 0; c < KS * 8; ++c) {
        const Halves s = split(x[c] * by);
        qf[n][0][c / 8][c % 8] = s.hi, qf[n][PARTS - 1][c / 8][c % 8] = s.lo;
      }
    }
  }
  if (tile < t_end) {
    load_k(tile, page);
    load_v(tile, page, v[0], vs[0]);
  }

  floatx4 acc[NT][CJ];
  float m_run[NT], l_run[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m_run[n] = NOTHING_SEEN;
    l_run[n] = 0.f;
#pragma unroll
    for (int j = 0; j < CJ; ++j) acc[n][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  auto turn = [&](auto more_tiles, auto buffer) __attribute__((always_inline)) {
    constexpr bool more = decltype(more_tiles)::value;
    constexpr int NOW = decltype(buffer)::value;
    floatx4 s[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < 2; ++m) s[n][m] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KS; ++c)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const half8 kf = operand_of<E4M3>(k[m][2 * c], k[m][2 * c + 1]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int x = 0; x < PARTS; ++x) s[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[n][x][c], s[n][m], 0, 0, 0);
      }
    const int ke = scale_exponent<k_scale_most<F32>()>(ks), ve = scale_exponent(vs[NOW]);
    if constexpr (more) {
      page = page_next;
      page_next = page_at(tile + 8);
      load_k(tile + 4, page);
      load_v(tile + 4, page, v[1 - NOW], vs[1 - NOW]);
    }
    const float k_by = exp2_int(ke), lift_v = (float)ve, v_back = exp2_int(-ve);
    const int t0 = tile * TT + 8 * g;
    if ((tile + 1) * TT > lim_min) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (t0 + 4 * m + r >= lim[n]) s[n][m][r] = -INFINITY;
    }
    half8 wf[NT][PARTS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float by = factor_of(k_by, q_scale[n]);
      float top = s[n][0][0];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[n][m][r]);
      const float mine = fmaf(top, by, lift_v);
      top = column_max(mine);
      const float ref = fmaxf(m_run[n], lifted(top, LIFT));
      if (__any(ref > m_run[n])) {
        const float shrink = exp2_fast(m_run[n] - ref);
        l_run[n] = add_scaled(0.f, l_run[n], m_run[n] - ref);
#pragma unroll
        for (int j = 0; j < CJ; ++j) acc[n][j] *= shrink;
        m_run[n] = ref;
      }
      float sum = 0.f;
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = exp2_fast(fmaf(s[n][m][r], by, lift_v - ref));
          sum += x;
          if constexpr (F32) {
            const Halves y = split(x);
            wf[n][0][4 * m + r] = y.hi, wf[n][PARTS - 1][4 * m + r] = y.lo;
          } else {
            wf[n][0][4 * m + r] = (half_t)x;
          }
        }
      float back = v_back;
      if constexpr (F32) {
        const bool far = mine - ref < FAR && mine > NOTHING_SEEN;
        if (__any(far)) {                                 // (before the weights it takes more registers: 2 x 16 heads of 1024 tokens 55 us, not 51)
          float y = 0.f;
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) y += exp2_fast(fmaf(s[n][m][r], by, FAR_LIFT - ref));
          sum = far ? y : sum, back = far ? exp2_int(-FAR_LIFT) : back;
        }
      }
      l_run[n] = fmaf(sum, back, l_run[n]);
    }
#pragma unroll
    for (int x = 0; x < VW; ++x) {
      unsigned lo[4], hi[4];
      {
        const unsigned r0[4] = {v[NOW][0][x], v[NOW][1][x], v[NOW][2][x], v[NOW][3][x]};
        const unsigned r1[4] = {v[NOW][4][x], v[NOW][5][x], v[NOW][6][x], v[NOW][7][x]};
        transpose4(r0, lo);
        transpose4(r1, hi);
      }
#pragma unroll
      for (int j = 0; j < (CJ < 4 ? CJ : 4); ++j) {
        const half8 vt = operand_of<E4M3>(lo[j], hi[j]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int y = 0; y < PARTS; ++y) acc[n][4 * x + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, wf[n][y], acc[n][4 * x + j], 0, 0, 0);
      }
    }
  };
  typedef std::integral_constant<int, 0> B0;
  typedef std::integral_constant<int, 1> B1;
  for (; tile + 8 < t_end; tile += 8) {
    turn(std::true_type(), B0());
    tile += 4;
    turn(std::true_type(), B1());
    tile -= 4;
  }
  if (tile + 4 < t_end) {
    turn(std::true_type(), B0());
    tile += 4;
    turn(std::false_type(), B1());
  } else if (tile < t_end) {
    turn(std::false_type(), B0());
  }

  // the four waves' states joined, and rows out: finished ones to `out`, the states of a slice to the workspace
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l_run[n] = column_sum(l_run[n]);
    if (g == 0) {
      box_m[w][n * 16 + i] = m_run[n];
      box_l[w][n * 16 + i] = l_run[n];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float o[CJ];
#pragma unroll
      for (int j = 0; j < CJ; ++j) o[j] = acc[n][j][r];
      store_words<CJ>(boxes[w] + (n * 16 + i) * LDB + (4 * g + r) * CJ, o);
    }
  }
  __syncthreads();
  for (int u = threadIdx.x; u < RB * (D / 4); u += 256) {
    const int at = u / (D / 4), e = u % (D / 4) * 4, row = rb * RB + at;
    const int iq = a.by_group.div(row), gq = row - iq * (int)a.by_group.d;
    if (row >= a.R || iq >= nq) continue;
    const float m = fmaxf(fmaxf(box_m[0][at], box_m[1][at]), fmaxf(box_m[2][at], box_m[3][at]));
    float l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      l = add_scaled(l, box_l[x][at], box_m[x][at] - m);
      o += *reinterpret_cast<const floatx4 *>(boxes[x] + at * LDB + e) * exp2_fast(box_m[x][at] - m);
    }
    if (a.slices == 1) {
      const float inv = inverse_of(l);
      T y[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) y[x] = (T)(o[x] * inv);
      store_words<(int)sizeof(T)>(static_cast<T *>(a.out) + (((long)b * a.n_q + iq) * a.Hq + h * (int)a.by_group.d + gq) * D + e, y);
    } else {
      const long to = ((long)h * a.B * a.slices + number) * a.R + row;
      *reinterpret_cast<floatx4 *>(a.part + to * D + e) = o;
      if (e == 0) a.part_ml[to] = make_float2(m, l);
    }
  }
}

// ---- many query rows, half precision -----------------------------------------------------------------------------------
// As over a pool of rows (attend_prompt): 32x32x16 products, a wave takes 32 query rows, a workgroup 32 NW that share the tiles of
// 64 slots; the 32-slot half blocks are a pipeline of logits, weights and outputs.  A tile's codes come to registers a turn ahead
// and are written to LDS as halves, once for all waves; so every turn has, beside its products, the codes of one tile of K and
// one of V to convert (16 codes: 20 vector instructions from int8, 8 from e4m3).
// Bound by LDS reads that products wait for and by vector instructions, with two waves a SIMD to cover for each other: 8 x 32 heads of
// 2048 tokens, d = 128, 376 us = 730 TFLOP/s of what is seen (the same over halves 351; without its LDS reads it would be 268);
// page_stream in blocks of 32 rows: 993.
// A wave's loads of a tile cover at most 16 consecutive slots, i.e. one page.  Lane l looks after the 16 slots
// l % 4 of a tile: their entry of the table (asked for three turns ahead), and their scales.
constexpr float RISE = 6.f, PROMPT_LIFT = 9.f;
constexpr int PROMPT_KEYS = 64;

template <int D, int NW, int RB, bool E4M3> __global__ __launch_bounds__(NW * 64, D * RB <= 128 ? 2 : 1) void page_prompt(StreamArgs a, PageRefs p) {
  constexpr int KS = D / 16, OB = D / 32, TK = PROMPT_KEYS, ROWS = RB * NW * 32;
  constexpr int LB = TK * D / (NW * 64) < 16 ? 8 : 16;            // bytes of a lane's load
  constexpr int PIECES = D / LB, LR = 64 / PIECES, LOADS = TK / (LR * NW);      // loads of a row; rows of a wave's load; loads of a wave
  static_assert(LOADS >= 1 && 16 % (LR * LOADS) == 0, "a wave's loads of a tile stay in a page");
  constexpr int LW = LB / 4;
  __shared__ __attribute__((aligned(16))) half_t tiles[2][2][TK * D];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 31, hb = lane >> 5;
  int work = xcd_order(blockIdx.x, a.per_xcd);
  if (work >= a.total) return;
  const int h = a.by_pair.div(work);
  work -= h * (int)a.by_pair.d;
  const int number = a.by_units.div(work), unit = a.by_units.mod(work);
  const Span span = span_of<false>(a, number);
  if (span.b < 0) return;
  const int b = span.b, slice = span.slice, G = (int)a.by_group.d, kv = span.kv, nq = span.nq;
  const int32_t *table = p.table + (long)b * p.stride;
  const unsigned in_page = (1u << p.shift) - 1;
  const unsigned long head = ((unsigned long)h << p.shift) * D;

  // where this lane's loads go: rows from_row, from_row + LR, .. of a tile, as halves from channel (lane % PIECES) LB on
  const int from_row = w * LR * LOADS + lane / PIECES, from_byte = lane % PIECES * LB;
  // (addresses of other pieces and columns are the first one's and a constant)
  const unsigned k_first = row_offset<D>(lane, 0), v_first = column_offset<D>(lane, 0, 0);

  for (int turn = 0; turn < (a.paired ? 2 : 1); ++turn) {
    const int rb = turn ? unit : a.nrb - 1 - unit;        // (a prompt's last rows see most: first)
    if (turn) {
      if (2 * unit >= a.nrb - 1) break;
      __syncthreads();                                    // the other waves are done with the tiles
    }
    int lim[RB], lim_min[RB];
    long row_at[RB];
    bool live[RB];
    half8 qf[RB][KS];
#pragma unroll
    for (int c = 0; c < RB; ++c) {
      const int first_row = rb * ROWS + (c * NW + w) * 32, row = first_row + i, iq = a.by_group.div(row), gq = row - iq * G;
      live[c] = row < a.R && iq < nq;
      lim[c] = live[c] ? row_limit<false>(a, row, kv, nq) : 0x7fffffff;
      lim_min[c] = row_limit<false>(a, first_row, kv, nq);
      row_at[c] = (((long)b * a.n_q + min(iq, a.n_q - 1)) * a.Hq + h * G + gq) * D;
      const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const half_t *>(a.q) + row_at[c]);
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[c][s] = __builtin_bit_cast(half8, flip_sign<half_t>(src[2 * s + hb], a.flip));
    }
    const int last_row = min(min(a.R, nq * G), (rb + 1) * ROWS) - 1;
    const int most = last_row < rb * ROWS ? 0 : row_limit<false>(a, last_row, kv, nq);
    const int tiles_all = (most + TK - 1) / TK;
    const int per = (tiles_all + span.slices - 1) / span.slices;
    const int t_begin = min(tiles_all, slice * per), t_end = min(tiles_all, t_begin + per);

    // (slots past the last one that a row sees are read from that one; tiles past the last: the last)
    const int last = most - 1;
    auto entry_of = [&](int tile) __attribute__((always_inline)) {
      return page_read(p, table[min(tile * TK + 16 * (lane & 3), last) >> p.shift]);
    };
    auto load_codes = [&](const char *pool, int tile, unsigned entries, unsigned (&to)[LOADS][LW]) __attribute__((always_inline)) {
      tile = min(tile, t_end - 1);
      const unsigned page = (unsigned)__builtin_amdgcn_readlane((int)entries, w * LR * LOADS / 16);
      const char *base = pool + (unsigned long)page * p.page_bytes + head;
#pragma unroll
      for (int x = 0; x < LOADS; ++x)
        load_words<LW>(base + (unsigned)((min(tile * TK + from_row + x * LR, last) & in_page) * D + from_byte), to[x]);
    };
    // part `x` of eight of a tile's codes to LDS as halves
    constexpr int RUNS = LOADS * LW / 2;                  // runs of eight codes that a lane holds
    auto store_halves = [&](int x, const unsigned (&from)[LOADS][LW], half_t *to) __attribute__((always_inline)) {
#pragma unroll
      for (int u = x * RUNS / 8; u < (x + 1) * RUNS / 8; ++u) {
        const int l = u / (LW / 2), y = u % (LW / 2), r = from_row + l * LR;
        *reinterpret_cast<half8 *>(reinterpret_cast<char *>(to) + r * D * 2 + ((from_byte / 8 + y) ^ piece_swap<D>(r)) * 16) =
            operand_of<E4M3>(from[l][2 * y], from[l][2 * y + 1]);
      }
    };

    floatx16 acc[RB][OB], sA[RB], sB[RB];
    float ref[RB], sum_all[RB];
    half8 pA[RB][2], pB[RB][2];
#pragma unroll
    for (int c = 0; c < RB; ++c) {
      ref[c] = NOTHING_SEEN, sum_all[c] = 0.f, sA[c] = floatx16{}, sB[c] = floatx16{};
#pragma unroll
      for (int o = 0; o < OB; ++o) acc[c][o] = floatx16{};
    }
    // of the lane's 16 slots of a tile: the factor of logits, the exponent of V's scale and 1 / that scale
    struct Scales {
      float k, v, back;
    };

    // now: logits in, weights out (half `now_half` of tile `now_tile`); next: the logits of rows `next_row` .. of tile K; out: acc +=
    // the weights `old` times rows `old_row` .. of tile V
    auto half_step = [&](auto has_now, auto has_next, auto has_old, const floatx16 (&now)[RB], int now_tile, auto now_half, const Scales &scales,
                         half8 (&weights)[RB][2], floatx16 (&next)[RB], const half_t *K, int next_row, const half8 (&old)[RB][2],
                         const half_t *V, int old_row, auto store) __attribute__((always_inline)) {
      constexpr bool NOW = decltype(has_now)::value, NEXT = decltype(has_next)::value, OLD = decltype(has_old)::value;
      constexpr int HALF = decltype(now_half)::value;
      // (operands are read LEAD products ahead: all at once they take more registers than there are)
      constexpr int LEAD = 3;
      half8 kf[KS];
      uint4 vt[2 * OB];
      const unsigned k_at = opaque(k_first), v_at = opaque(v_first);
      auto read = [&](int x) __attribute__((always_inline)) {
        if constexpr (NEXT) {
#pragma unroll
          for (int k = x * KS / 8; k < (x + 1) * KS / 8; ++k) kf[k] = row_piece(K + next_row * D, k_at ^ k << 5);
        }
        if constexpr (OLD) {
#pragma unroll
          for (int y = x * 2 * OB / 8; y < (x + 1) * 2 * OB / 8; ++y) {
            const half_t *rows = V + (old_row + y / OB * 16) * D;
            const uint2 lo = column_rows<D>(rows, v_at ^ y % OB << 6, 0), hi = column_rows<D>(rows, v_at ^ (y % OB << 6 | 1 << 5), 1);
            vt[y] = make_uint4(lo.x, lo.y, hi.x, hi.y);
          }
        }
      };
#pragma unroll
      for (int x = 0; x < LEAD; ++x) read(x);
      floatx16 s[RB];
      float shrink[RB], by[2], off[RB][2], back[2], sums[RB][4] = {};
      bool rises[RB];
      if constexpr (NOW) {
        float exponent[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          auto of = [&](float y) __attribute__((always_inline)) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(y), HALF * 2 + x)); };
          by[x] = of(scales.k), exponent[x] = of(scales.v), back[x] = of(scales.back);
        }
#pragma unroll
        for (int c = 0; c < RB; ++c) {
          s[c] = now[c];
          const int t0 = now_tile * TK + HALF * 32;
          if (t0 + 32 > lim_min[c]) {
            const int mine = t0 + (int)opaque(hb * 4);
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (mine + ((e / 4) * 8 + e % 4) >= lim[c]) s[c][e] = -INFINITY;
          }
        }
#pragma unroll
        for (int c = 0; c < RB; ++c) {
          float top = -INFINITY;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float m = s[c][8 * x];
#pragma unroll
            for (int e = 8 * x + 1; e < 8 * x + 8; ++e) m = __builtin_elementwise_maximum(m, s[c][e]);
            top = fmaxf(top, fmaf(m, by[x], exponent[x]));
          }
          top = lifted(both_max(top), PROMPT_LIFT);
          const float to = top > ref[c] + RISE ? top : ref[c];
          rises[c] = __any(to != ref[c]);
          shrink[c] = exp2_fast(ref[c] - to);
          ref[c] = to;
          sum_all[c] *= shrink[c];
#pragma unroll
          for (int x = 0; x < 2; ++x) off[c][x] = exponent[x] - to;
        }
      }
      if constexpr (NEXT) {
#pragma unroll
        for (int c = 0; c < RB; ++c) next[c] = floatx16{};
      }
      __builtin_amdgcn_s_setprio(1);                      // (a wave that multiplies before one that works out references: half a percent)
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        if (x + LEAD < 8) read(x + LEAD);
        store(x);
        if constexpr (NEXT) {
#pragma unroll
          for (int k = x * KS / 8; k < (x + 1) * KS / 8; ++k)
#pragma unroll
            for (int c = 0; c < RB; ++c) next[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[k], qf[c][k], next[c], 0, 0, 0);
        }
        if constexpr (OLD) {
#pragma unroll
          for (int y = x * 2 * OB / 8; y < (x + 1) * 2 * OB / 8; ++y)
#pragma unroll
            for (int c = 0; c < RB; ++c)
              acc[c][y % OB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, vt[y]), old[c][y / OB], acc[c][y % OB], 0, 0, 0);
        }
        if constexpr (NOW) {
#pragma unroll
          for (int c = 0; c < RB; ++c)
#pragma unroll
            for (int e = 2 * x; e < 2 * x + 2; ++e) {
              const float y = exp2_fast(fmaf(s[c][e], by[e / 8], off[c][e / 8]));
              sums[c][e / 8 * 2 + e % 2] += y;
              weights[c][e / 8][e % 8] = (half_t)y;
            }
        }
      }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (NOW) {
#pragma unroll
        for (int c = 0; c < RB; ++c) {
          sum_all[c] = fmaf(sums[c][0] + sums[c][1], back[0], fmaf(sums[c][2] + sums[c][3], back[1], sum_all[c]));
          keep_here(weights[c][0]);
          keep_here(weights[c][1]);
          keep_here(sum_all[c]);                          // (not put off: the weights' registers are needed)
        }
#pragma unroll
        for (int c = 0; c < RB; ++c)
          if (rises[c]) {
#pragma unroll
            for (int o = 0; o < OB; ++o) acc[c][o] *= shrink[c];
          }
      }
    };
    typedef std::true_type Y;
    typedef std::false_type N;
    typedef std::integral_constant<int, 0> H0;
    typedef std::integral_constant<int, 1> H1;
    if (t_end > t_begin) {
      const int turns = t_end - t_begin;
      unsigned k_codes[LOADS][LW], v_codes[LOADS][LW];
      // entries of the tile that K is asked for next, and of the one after it; scales of this turn's tile, the last one's and the next
      unsigned e0 = entry_of(t_begin), e1 = entry_of(t_begin + 1), e2 = entry_of(t_begin + 2);
      auto scales_of = [&](unsigned entry) __attribute__((always_inline)) {
        const unsigned long at = (unsigned long)entry * p.H + h;
        return make_float2(p.K_scale[at], p.V_scale[at]);
      };
      auto ready = [&](float2 s) __attribute__((always_inline)) {
        const int ke = scale_exponent<k_scale_most<false>()>(s.x), ve = scale_exponent(s.y);
        return Scales{factor_of(exp2_int(ke), a.c), (float)ve, exp2_int(-ve)};
      };
      Scales now = ready(scales_of(e0)), before = now;
      float2 ahead;
      load_codes(p.K, t_begin, e0, k_codes);
#pragma unroll
      for (int x = 0; x < 8; ++x) store_halves(x, k_codes, tiles[0][0]);
      load_codes(p.K, t_begin + 1, e1, k_codes);
      load_codes(p.V, t_begin, e0, v_codes);
      ahead = scales_of(e1);
      // Turn r: tile r of K is in slot r % 2, r - 1 of V in the other one; the codes of K r + 1 and V r are in registers and go to the
      // free slots among the products, K's in the first half, V's in the second.
      auto to_slot = [&](const unsigned (&codes)[LOADS][LW], half_t *to) __attribute__((always_inline)) {
        return [&codes, to, &store_halves](int x) __attribute__((always_inline)) { store_halves(x, codes, to); };
      };
      auto nothing = [](int) __attribute__((always_inline)) {};
      auto middle = [&](int r) __attribute__((always_inline)) { load_codes(p.K, t_begin + r + 2, e2, k_codes); };
      auto end_turn = [&](int r) __attribute__((always_inline)) {
        load_codes(p.V, t_begin + r + 1, e1, v_codes);
        e1 = e2;
        e2 = entry_of(t_begin + r + 3);
        before = now, now = ready(ahead);
        ahead = scales_of(e1);
        __syncthreads();                                  // the next turn's tiles are there, and the other slots are free
      };
      auto turn_of = [&](int r, auto slot) __attribute__((always_inline)) {
        constexpr int S = decltype(slot)::value;
        const half_t *K = tiles[S][0], *V = tiles[1 - S][1];
        half_step(Y(), Y(), Y(), sB, t_begin + r - 1, H1(), before, pB, sA, K, 0, pA, V, 0, to_slot(k_codes, tiles[1 - S][0]));
        middle(r);
        half_step(Y(), Y(), Y(), sA, t_begin + r, H0(), now, pA, sB, K, 32, pB, V, 32, to_slot(v_codes, tiles[S][1]));
        end_turn(r);
      };
      __syncthreads();
      half_step(N(), Y(), N(), sB, 0, H0(), now, pB, sA, tiles[0][0], 0, pA, tiles[0][1], 0, to_slot(k_codes, tiles[1][0]));
      middle(0);
      half_step(Y(), Y(), N(), sA, t_begin, H0(), now, pA, sB, tiles[0][0], 32, pB, tiles[0][1], 0, to_slot(v_codes, tiles[0][1]));
      end_turn(0);
      int r = 1;
      // (tested at its end: tested at its beginning the compiler keeps outputs and logits twice, 75 registers more)
      if (r + 1 < turns) do {
        turn_of(r, H1());
        turn_of(r + 1, H0());
        r += 2;
      } while (r + 1 < turns);
      if (r < turns) turn_of(r, H1());
      const half_t *V = tiles[(turns - 1) % 2][1];
      half_step(Y(), N(), Y(), sB, t_end - 1, H1(), before, pB, sA, V, 0, pA, V, 0, nothing);
      half_step(N(), N(), Y(), sA, 0, H0(), now, pA, sB, V, 0, pB, V, 32, nothing);
    }

#pragma unroll
    for (int c = 0; c < RB; ++c) {
      const float sum = both_sum(sum_all[c]);
      if (!live[c]) continue;
      const float inv = inverse_of(sum);
      if (a.slices == 1) {
        half_t *to = static_cast<half_t *>(a.out) + row_at[c];
#pragma unroll
        for (int o = 0; o < OB; ++o)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            half_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (half_t)(acc[c][o][x * 4 + e] * inv);
            store_words<2>(to + o * 32 + x * 8 + hb * 4, v);
          }
      } else {
        const long at = ((long)h * a.B * a.slices + number) * a.R + rb * ROWS + (c * NW + w) * 32 + i;
#pragma unroll
        for (int o = 0; o < OB; ++o)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            *reinterpret_cast<floatx4 *>(a.part + at * D + o * 32 + x * 8 + hb * 4) =
                floatx4{acc[c][o][x * 4], acc[c][o][x * 4 + 1], acc[c][o][x * 4 + 2], acc[c][o][x * 4 + 3]};
        if (hb == 0) a.part_ml[at] = make_float2(ref[c], sum);
      }
    }
  }
}

int div_up(long n, long d) { return (int)((n + d - 1) / d); }

// Query rows of a workgroup: page_stream's 16 or 32, page_prompt's 128 or 256 (as over a pool of rows, by the same rules).
// In float32 32 only where turns of 128 slots are enough to fill the GPU with (whole calls, d = 128: 2 x 16 heads of 1024 tokens 51
// us with 32, 55 with 16; 20 rows, 16 x 8 of 4096, 39 and 48; but 4 heads of 512 13.7 and 10.0).
int row_block(const ig_desc *d, long R) {
  if (R <= 16 || d->d > 128) return 16;
  return d->dtype == IG_F16 || (double)d->B * d->H * div_up(R, 32) * div_up(d->N, 128) >= 1024 ? 32 : 16;
}
// page_stream's row blocks read the codes again for every 32 (d = 256: 16) rows, out of the caches, page_prompt's 128 once, but a turn of
// its takes longer.  (16 x 8 heads of 4096, 40 rows: 47 us there, 53 here; d = 64, 48 rows 32 and 35; d = 256, 20 rows 75 and
// 115, 60 rows, 4 x 8 of 4000, 45 and 50; 56 rows, 3 x 11 ragged of 4923, 23 and 26; but 72 rows, 16 x 8 of 4096, 66 and 59.
// Where a few heads leave the GPU mostly empty page_stream is the faster one beyond 64 rows, too: a sequence of 1000 slots, d = 128, 256 rows of 1, 4
// and 8 heads 12, 13 and 19 us, page_prompt 17, 18 and 20; 512 rows of 8 heads over 4096 33 and 33.)
bool many_rows(const ig_desc *d, long R) { return d->dtype == IG_F16 && R > 64; }
// page_prompt's: at d = 128 eight waves or four.  Eight where most of what the rows see is seen by all of them (317 x 4 query rows
// over up to 9001, 4 x 8 heads: 197 us, 206 with four), four for prompts, where a block of 256 rows works out more that its first
// rows do not see (2048 over 2048, 8 x 32 heads: 380 us, 394 with eight; no difference with 4 x 8 heads of 4 query heads each).  At
// d = 64 two row blocks a wave or one: two where workgroups enough are left (2048 over 2048, 4 x 32 heads 113 us, 123 with one;
// 4 x 16 of 2 query heads each 106 and 117), one where not (317 x 4 over up to 9001, 4 x 8 heads: 116 us, 125 with two).
int prompt_rows(const ig_desc *d, const PageCall &c) {
  const long R = (long)c.n_q * c.group;
  if (d->d == 128) return R > 128 && 2 * (long)c.n_q <= d->N ? 256 : 128;
  return d->d == 64 && d->B * (long)d->H * div_up(R, 256) >= 512 ? 256 : 128;
}
int page_waves(const ig_desc *d, int rb) { return rb == 256 && d->d == 128 ? 8 : 4; }

// Slices that the slots of a pool head are cut into: the number for which the last workgroups end first.  page_prompt: as over a
// pool of rows.  page_stream, in turns of 128 slots: the fullest compute unit has n workgroups, which take turns two at a time, and
// 4/5 of a turn each where memory is what holds them up; four turns to start, and for a join two and three for every eight
// slices.  (8 x 32 heads of 2048: 31 us with 1 slice, 35 with 2, 38 with 4; 32 of 777: 8.5 with 7, 10.3 with 1; 4 x 8 of 8192:
// 18 with 8, 22 with 4; 16 x 8 ragged of 32768: 131 with 4, 159 with 3, 177 with 2.)
// Never more than four rounds of workgroups, so that the states they leave are bounded (ig_page_reserve_bytes).
constexpr long ROUNDS = 4;
long workgroups_of(int rb) { return rb == 256 ? 256 : 512; }
int slices_of(const ig_desc *d, const PagePlan &p) {
  const long groups = d->B * (long)d->H * p.nrb, turns = div_up(d->N, p.prompt ? 64 : 128), at_once = workgroups_of(p.rb);
  long best = 1, best_cost = -1;
  for (long s = 1; s <= MOST_SLICES && s <= turns && (s == 1 || groups * s <= ROUNDS * at_once); ++s) {
    const long per = div_up(turns, s), join = s > 1 ? 3 * div_up(s, 8) : 0;
    long cost = div_up(groups * s, at_once) * (per + 2) + join;
    if (!p.prompt) {
      const long n = div_up(groups * s, 256), two = 5 * div_up(n, 2) * per, bound = 4 * n * per;
      cost = (two > bound ? two : bound) + 5 * (4 + join + (s > 1 ? 2 : 0));
    }
    if (best_cost < 0 || cost < best_cost) best = s, best_cost = cost;
  }
  return (int)best;
}

}  // namespace

PagePlan ig_page_plan(const ig_desc *d, const PageCall &c) {
  PagePlan p = {};
  const long R = (long)c.n_q * c.group, BH = (long)d->B * d->H;
  p.prompt = many_rows(d, R);
  p.rb = p.prompt ? prompt_rows(d, c) : row_block(d, R);
  p.nrb = div_up(R, p.rb);
  p.slices = slices_of(d, p);
  p.threads = (BH * p.slices * p.nrb + 8) * 64 * page_waves(d, p.rb);
  const size_t ml = p.slices > 1 ? BH * p.slices * R * sizeof(float2) : 0;
  p.part_at = (ml + 255) / 256 * 256;
  p.bytes = p.part_at + (p.slices > 1 ? BH * p.slices * R * d->d * sizeof(float) : 0);
  return p;
}

// A bound for any number of tokens and slots up to these: states of at most MOST_SLICES slices of every row, and of at most
// ROUNDS rounds of workgroups.
size_t ig_page_reserve_bytes(const ig_desc *d, int group, int n_q) {
  const long all = (long)MOST_SLICES * d->B * d->H * n_q * group, rounds = ROUNDS * (d->dtype == IG_F16 ? 256 * workgroups_of(256) : 32 * workgroups_of(32));
  return (size_t)(all < rounds ? all : rounds) * (sizeof(float2) + d->d * sizeof(float)) + 2 * 256;
}

int ig_launch_page_attention(ig_ctx *ctx, const ig_desc *d, const ig_pages *pages, const PageCall &c, const PagePlan &p, char *ws, hipStream_t stream) {
  const long BH = (long)d->B * d->H;
  const PageRefs refs = ig_page_refs(d, pages);
  StreamArgs a = {};
  a.q = c.q, a.out = c.out, a.q_len = c.q_len, a.kv_len = c.kv_len;
  a.n_q = c.n_q, a.R = c.n_q * c.group, a.Hq = d->H * c.group, a.N = d->N, a.N_cap = d->N_cap;
  a.nrb = p.nrb, a.slices = p.slices, a.B = d->B, a.H = d->H, a.turn_shift = !p.prompt;
  a.by_slices = ig_fast_div(p.slices), a.by_H = ig_fast_div(d->H), a.by_group = ig_fast_div(c.group);
  a.flip = d->scale < 0.f ? 1 : (d->scale == 0.f ? 2 : 0);
  a.c = (d->scale == 0.f ? 1.f : fabsf(d->scale)) * 1.44269504088896340736f;
  a.part_ml = reinterpret_cast<float2 *>(ws);
  a.part = reinterpret_cast<float *>(ws + p.part_at);
  // a causal call with workgroups to spare: each takes a late and an early row block, so that all take equally long
  a.paired = p.prompt && p.slices == 1 && BH * p.nrb >= 1024 && 2 * c.n_q > d->N;
  const int units = a.paired ? (p.nrb + 1) / 2 : p.nrb;
  a.by_units = ig_fast_div(units), a.by_pair = ig_fast_div(d->B * p.slices * units);
  a.total = (int)(BH * p.slices * units), a.per_xcd = div_up(a.total, 8);
  const dim3 grid(a.per_xcd * 8), block(256);
#define STREAM(D, NT, E4M3, F32, ONCE)                                                               \
  {                                                                                                  \
    auto k = page_stream<D, NT, E4M3, F32, ONCE>;                                                    \
    IG_LAUNCH(ctx, IG_K_CACHE, k, grid, block, stream, a, refs);                                     \
  }
#define STREAM_ONCE(D, NT, E4M3, F32)                                                                \
  {                                                                                                  \
    if (p.nrb == 1) STREAM(D, NT, E4M3, F32, true) else STREAM(D, NT, E4M3, F32, false)              \
  }
#define PROMPT_WAVES(D, NW, RB, E4M3)                                                                \
  {                                                                                                  \
    auto k = page_prompt<D, NW, RB, E4M3>;                                                           \
    IG_LAUNCH(ctx, IG_K_CACHE, k, grid, dim3(NW * 64), stream, a, refs);                             \
  }
#define PROMPT(D, E4M3)                                                                              \
  {                                                                                                  \
    if (p.rb == 128) PROMPT_WAVES(D, 4, 1, E4M3)                                                     \
    else if constexpr (D == 64) PROMPT_WAVES(D, 4, 2, E4M3)                                          \
    else if constexpr (D == 128) PROMPT_WAVES(D, 8, 1, E4M3)                                         \
  }
#define STREAM_ROWS(D, E4M3)                                                                         \
  {                                                                                                  \
    if (p.rb == 16 && d->dtype == IG_F32) STREAM_ONCE(D, 1, E4M3, true)                              \
    else if (p.rb == 16) STREAM_ONCE(D, 1, E4M3, false)                                              \
    else if constexpr (D <= 128) {                                                                   \
      if (d->dtype == IG_F32) STREAM_ONCE(D, 2, E4M3, true) else STREAM_ONCE(D, 2, E4M3, false)      \
    }                                                                                                \
  }
#define BY_DIM(DO, E4M3)                                                                             \
  switch (d->d) {                                                                                    \
    case 32: DO(32, E4M3) break;                                                                     \
    case 64: DO(64, E4M3) break;                                                                     \
    case 128: DO(128, E4M3) break;                                                                   \
    default: DO(256, E4M3) break;                                                                    \
  }
  if (p.prompt) {
    if (pages->code == IG_CODE_I8) BY_DIM(PROMPT, false) else BY_DIM(PROMPT, true)
  } else {
    if (pages->code == IG_CODE_I8) BY_DIM(STREAM_ROWS, false) else BY_DIM(STREAM_ROWS, true)
  }
  return p.slices > 1 ? ig_launch_join(ctx, d, a, nullptr, stream) : IG_OK;
}
