// Rotary embedding of rows, their append to pages of 8-bit codes with a scale for each page and head, and rows read back.
#include "page_device.h"

namespace {

int div_up(long n, long d) { return (int)((n + d - 1) / d); }

// ---- rotation ------------------------------------------------------------------------------------------------------
// A thread takes one unit of a token, works out its eight turns once, and takes `per` heads of it, the next head's values asked
// for ahead.  Bound by memory: 16 x 2048 tokens of 32 heads, d = 128, 102 us = 5.3 TB/s (a copy of 2 GiB: 4.7); one token 2.8 us, of
// which a launch is two.
struct RotateArgs {
  const void *x;
  void *out;
  const int32_t *pos;
  long x_stride, out_stride;
  int heads, per, d;
  int total;                          // units of all tokens, times their parts of `per` heads
  FastDiv by_units, by_parts;
  RotaryRefs r;
};
template <typename T, int KIND>
__device__ __forceinline__ void rotate_heads(const T *x, T *out, int d, int h0, int h1, int s, int pos, const RotaryRefs &r) {
  Unit<T, KIND> u;
  u.load(x + (long)h0 * d, s, r.dims);
  float2 turn[8];
  if (KIND != TURN_NONE && 16 * s < r.dims) turns_of(s, pos, r, turn);
  for (int h = h0; h < h1; ++h) {
    float v[16];
    u.get(v);
    if (h + 1 < h1) u.load(x + (long)(h + 1) * d, s, r.dims);
    rotate_unit<KIND>(v, s, r.dims, turn);
    Unit<T, KIND>::store(out + (long)h * d, s, r.dims, v);
  }
}
template <typename T, int KIND> __global__ __launch_bounds__(256) void rotate_rows(RotateArgs a) {
  const int u = blockIdx.x * 256 + threadIdx.x;
  if (u >= a.total) return;
  const int at = a.by_units.div(u), s = u - at * (int)a.by_units.d, i = a.by_parts.div(at), h = (at - i * (int)a.by_parts.d) * a.per;
  rotate_heads<T, KIND>(static_cast<const T *>(a.x) + i * a.x_stride, static_cast<T *>(a.out) + i * a.out_stride, a.d, h, min(h + a.per, a.heads), s,
                  a.pos[i], a.r);
}

// ---- append --------------------------------------------------------------------------------------------------------
// A workgroup takes the new rows of one page of a sequence, of K or of V, head after head of `per`: two units of 16
// channels a thread, their turns worked out once for all heads, the next head's values asked for ahead.  The largest value
// of a head's rows gives the scale.  Rows stay in registers from their load to their codes, so that every byte passes once: 16 x
// 2048 rows of 32 heads with their queries, d = 128, 240 us = 5.6 TB/s (keys and values in one workgroup, without the next
// head ahead, spilled: 366).  One row of 16 sequences, 8 heads, 5.1 us: lengths, entry, and scale and rows are trips in turn.
constexpr int APPEND_UNITS = 2;
struct AppendArgs {
  PageRefs p;
  const void *q, *k, *v;
  void *q_out;
  const int32_t *n_append, *kv_len, *pos;
  long q_stride, kv_stride;
  int H, Hq, d, unit_shift, N, N_cap, n_rows;           // a row has 1 << unit_shift units
  int per, q_per;                     // heads of a workgroup, and of a thread that rotates queries
  int kv_blocks, q_total;             // workgroups of the pages; threads of those behind them, which rotate queries
  FastDiv by_pages, by_parts, by_rows, by_q_parts;      // pages that a sequence's rows touch at most, parts of `per` heads, ..
  RotaryRefs r;
};
// the value to be stored: 0 for one that is not finite
__device__ __forceinline__ float finite_or_zero(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.f : x; }

template <typename T, bool E4M3, int KIND> __device__ __forceinline__ void append_page(const AppendArgs &a, int kv, float (&tops)[2][16]) {
  const int tid = threadIdx.x, team = blockDim.x, work = blockIdx.x >> 1;
  const int at = a.by_pages.div(work), p = work - at * (int)a.by_pages.d, b = a.by_parts.div(at), h0 = (at - b * (int)a.by_parts.d) * a.per;
  const int start = a.kv_len ? min(max(a.kv_len[b], 0), a.N_cap) : a.N;
  const int n = min(a.n_append ? min(max(a.n_append[b], 0), a.n_rows) : a.n_rows, a.N_cap - start);
  const int number = (start >> a.p.shift) + p, slot0 = number << a.p.shift;
  const int r0 = max(start, slot0), r1 = min(start + n, slot0 + (1 << a.p.shift));
  if (r0 >= r1) return;
  const int entry = a.p.table[(long)b * a.p.stride + number];
  if ((unsigned)entry >= a.p.n_pages) return;
  const int held = r0 - slot0, total = (r1 - r0) << a.unit_shift, dims = kv ? 0 : a.r.dims;
  const int h1 = min(h0 + a.per, a.H);
  const T *rows = static_cast<const T *>(kv ? a.v : a.k) + ((long)b * a.n_rows + (r0 - start)) * a.kv_stride;
  float *scales = (kv ? a.p.V_scale : a.p.K_scale) + (long)entry * a.H;

  int row[APPEND_UNITS], unit[APPEND_UNITS];
  bool mine[APPEND_UNITS];
  Unit<T, KIND> in[APPEND_UNITS];
  float scale = 0.f;
  // (a thread without a unit reads the first row and stores nothing)
  auto ask = [&](int h) __attribute__((always_inline)) {
    if (held) scale = scales[h];
#pragma unroll
    for (int k = 0; k < APPEND_UNITS; ++k) in[k].load(rows + row[k] * a.kv_stride + (long)h * a.d, unit[k], dims);
  };
#pragma unroll
  for (int k = 0; k < APPEND_UNITS; ++k) {
    const int u = tid + k * team;
    mine[k] = u < total;
    row[k] = mine[k] ? u >> a.unit_shift : 0, unit[k] = u & ((1 << a.unit_shift) - 1);
  }
  ask(h0);
  float2 turn[APPEND_UNITS][8];
  if (KIND != TURN_NONE && dims) {
    const int first_pos = (a.pos ? a.pos[b] : start) + (r0 - start);
#pragma unroll
    for (int k = 0; k < APPEND_UNITS; ++k)
      if (mine[k] && 16 * unit[k] < dims) turns_of(unit[k], first_pos + row[k], a.r, turn[k]);
  }
  for (int h = h0; h < h1; ++h) {
    float x[APPEND_UNITS][16], top = 0.f;
    int before = held ? scale_exponent(scale) : SCALE_LEAST;
#pragma unroll
    for (int k = 0; k < APPEND_UNITS; ++k) in[k].get(x[k]);
    if (h + 1 < h1) ask(h + 1);
#pragma unroll
    for (int k = 0; k < APPEND_UNITS; ++k) {
      rotate_unit<KIND>(x[k], unit[k], dims, turn[k]);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[k][e] = finite_or_zero(x[k][e]);
        if (mine[k]) top = fmaxf(top, fabsf(x[k][e]));
      }
    }
    top = wave_max(top);
    if (team > 64) {
      if (tid % 64 == 0) tops[h & 1][tid / 64] = top;
      // (the scale is there before any thread may store a new one)
      asm volatile("" : "+v"(before));
      __syncthreads();
      for (int w = 0; w < team / 64; ++w) top = fmaxf(top, tops[h & 1][w]);
    }
    const int e2 = max(before, exponent_for<E4M3>(top));
    char *page = (kv ? a.p.V : a.p.K) + (unsigned long)(unsigned)entry * a.p.page_bytes + ((unsigned long)h << a.p.shift) * a.d;
    if (held && e2 > before) {
      const float by = exp2_int(max(before - e2, -126));
      for (int u = tid; u < held << a.unit_shift; u += team) {
        uint4 *c = reinterpret_cast<uint4 *>(page) + u;
        const uint4 v = *c;
        unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx4 f = decode4<E4M3>(w[i]) * by;
          w[i] = encode4<E4M3>(f[0], f[1], f[2], f[3]);
        }
        *c = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    const float inv = exp2_int(-e2);
#pragma unroll
    for (int k = 0; k < APPEND_UNITS; ++k) {
      if (!mine[k]) continue;
      char *to = page + (long)(held + row[k]) * a.d;
      unsigned c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = encode4<E4M3>(x[k][4 * i] * inv, x[k][4 * i + 1] * inv, x[k][4 * i + 2] * inv, x[k][4 * i + 3] * inv);
      Unit<T, KIND>::store_codes(to, unit[k], dims, c);
    }
    if (tid == 0 && (!held || e2 > before)) scales[h] = exp2_int(e2);
  }
}

template <typename T, bool E4M3, int KIND> __global__ __launch_bounds__(1024) void append_pages(AppendArgs a) {
  __shared__ float tops[2][16];
  if ((int)blockIdx.x >= a.kv_blocks) {
    const int u = (blockIdx.x - a.kv_blocks) * blockDim.x + threadIdx.x;
    if (u >= a.q_total) return;
    const int at = u >> a.unit_shift, s = u & ((1 << a.unit_shift) - 1), i = a.by_q_parts.div(at), h = (at - i * (int)a.by_q_parts.d) * a.q_per;
    const int b = a.by_rows.div(i), j = i - b * a.n_rows;
    if (j >= (a.n_append ? min(max(a.n_append[b], 0), a.n_rows) : a.n_rows)) return;
    const int first = a.pos ? a.pos[b] : (a.kv_len ? min(max(a.kv_len[b], 0), a.N_cap) : a.N);
    rotate_heads<T, KIND>(static_cast<const T *>(a.q) + i * a.q_stride, static_cast<T *>(a.q_out) + (long)i * a.Hq * a.d, a.d, h, min(h + a.q_per, a.Hq), s,
                    first + j, a.r);
    return;
  }
  // (values have no short runs)
  if (run_of(KIND) < 8 && (blockIdx.x & 1)) append_page<T, E4M3, TURN_NONE>(a, 1, tops);
  else append_page<T, E4M3, KIND>(a, blockIdx.x & 1, tops);
}

// ---- rows read back ------------------------------------------------------------------------------------------------
// A thread takes the channels of one 16-byte store, of GATHER_ROWS listed rows of K and of V, all entries and then all codes
// asked for together.  Stores are past the caches: whole lines of rows that somebody else reads.  Bound by memory: 160 lists of
// 1638, d = 128, 35 us = 5.1 TB/s (16 codes a thread, one row, stores through the caches: 44; four rows: 38); 256 of 102, 5.0 us.
constexpr int GATHER_ROWS = 2;
struct GatherArgs {
  PageRefs p;
  const int32_t *sel_idx, *sel_cnt;
  void *K_sel, *V_sel;
  int H, N_cap, sel_stride;
  FastDiv by_chunks, by_H;
};
template <typename T, int D, bool E4M3> __global__ __launch_bounds__(256) void gather_pages(GatherArgs a) {
  constexpr int CH = 16 / (int)sizeof(T), UNITS = D / CH, STEP = 256 / UNITS, U = GATHER_ROWS;
  typedef unsigned codes_t __attribute__((ext_vector_type(CH / 4)));
  typedef T vec __attribute__((ext_vector_type(CH)));
  const int bh = a.by_chunks.div(blockIdx.x), chunk = blockIdx.x - bh * (int)a.by_chunks.d, b = a.by_H.div(bh), h = bh - b * a.H;
  const int n = min(a.sel_cnt[bh], a.sel_stride), j0 = chunk * STEP * U + threadIdx.x / UNITS, s = threadIdx.x % UNITS;
  if (j0 >= n) return;
  int slot[U];
  unsigned page[U];
#pragma unroll
  for (int u = 0; u < U; ++u) slot[u] = min(max(a.sel_idx[(long)bh * a.sel_stride + min(j0 + u * STEP, n - 1)], 0), a.N_cap - 1);
#pragma unroll
  for (int u = 0; u < U; ++u) page[u] = page_read(a.p, a.p.table[(long)b * a.p.stride + (slot[u] >> a.p.shift)]);
  codes_t codes[U][2];
  float scale[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const unsigned long from = (unsigned long)page[u] * a.p.page_bytes + (((unsigned long)h << a.p.shift) + (slot[u] & ((1 << a.p.shift) - 1))) * D + s * CH;
    codes[u][0] = *reinterpret_cast<const codes_t *>(a.p.K + from), codes[u][1] = *reinterpret_cast<const codes_t *>(a.p.V + from);
    scale[u][0] = a.p.K_scale[(long)page[u] * a.H + h], scale[u][1] = a.p.V_scale[(long)page[u] * a.H + h];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (j0 + u * STEP >= n) break;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const float by = exp2_int(scale_exponent(scale[u][kv]));
      vec x;
#pragma unroll
      for (int i = 0; i < CH / 4; ++i) {
        const floatx4 f = decode4<E4M3>(codes[u][kv][i]) * by;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i + e] = (T)f[e];
      }
      T *to = static_cast<T *>(kv ? a.V_sel : a.K_sel) + ((long)bh * a.sel_stride + j0 + u * STEP) * D + s * CH;
      __builtin_nontemporal_store(x, reinterpret_cast<vec *>(to));
    }
  }
}

// Heads that are taken one after the other, so that turns are worked out once for them: one where that is what fills the GPU
// with waves, up to eight where there are enough.  (One and eight.  The kernel alone: a row each for 16 ragged sequences of 8 heads
// with their 4 query heads each, 5.0 and 12.7 us; 317 rows each for 3 ragged sequences of 12 heads of 64 in float32, 7.3 and 14.1;
// one row of 4 heads rotated 2.7 and 3.4.  The whole call: 2048 rows each for 16 x 32 heads 611 and 408 us, rotated alone 126 and 102.)
int heads_each(int heads, double threads) {
  int per = 1;
  while (per < 8 && per < heads && threads / (2 * per) >= 65536.0) per *= 2;
  return per;
}
// Pages that n_rows new rows of a sequence touch at most, and threads of a workgroup: a page's new rows in two units each.
int append_page_count(const ig_pages *p, int n_rows) { return (n_rows + p->page_size - 2) / p->page_size + 1; }
int append_team(const ig_desc *d, const ig_pages *p, int n_rows) {
  const int units = (n_rows < p->page_size ? n_rows : p->page_size) * d->d / 16;
  int team = 64;
  while (team * APPEND_UNITS < units) team *= 2;
  return team;
}

int rotate_each(long n, int heads, int d) { return heads_each(heads, (double)n * heads * (d / 16)); }
int append_each(const ig_desc *d, const ig_pages *p, int n_rows) {
  return heads_each(d->H, 2.0 * d->B * append_page_count(p, n_rows) * d->H * append_team(d, p, n_rows));
}

// An append's launch: workgroups of `team` threads for the new rows of a page, of K or of V, and behind them those that rotate queries.
struct AppendGrid {
  int pages, per, parts, q_per, q_parts, team;
  long kv_blocks, q_total;            // (at most 2^27 and 2^30: there are at most 2^26 rows, of queries too)
};
AppendGrid append_grid(const ig_desc *d, const ig_pages *p, int Hq, int n_rows) {
  AppendGrid g;
  const long n = (long)d->B * n_rows;
  g.pages = append_page_count(p, n_rows), g.team = append_team(d, p, n_rows);
  g.per = append_each(d, p, n_rows), g.q_per = Hq ? rotate_each(n, Hq, d->d) : 1;
  g.parts = div_up(d->H, g.per), g.q_parts = Hq ? div_up(Hq, g.q_per) : 1;
  g.kv_blocks = 2l * d->B * g.pages * g.parts, g.q_total = Hq ? n * g.q_parts * (d->d / 16) : 0;
  return g;
}

}  // namespace

long ig_append_pages_threads(const ig_desc *d, const ig_pages *p, int Hq, int n_rows) {
  const AppendGrid g = append_grid(d, p, Hq, n_rows);
  return (g.kv_blocks + div_up(g.q_total, g.team)) * g.team;
}

long ig_rotate_threads(int n, int heads, int d) { return (long)n * div_up(heads, rotate_each(n, heads, d)) * (d / 16) + 255; }

int ig_launch_rotate(ig_ctx *ctx, int dtype, int n, int heads, int d, const ig_rotary *rotary, int inverse, const int32_t *pos, const void *x,
                     long x_stride, void *out, long out_stride, hipStream_t s) {
  RotateArgs a = {};
  a.x = x, a.out = out, a.pos = pos, a.x_stride = x_stride, a.out_stride = out_stride, a.heads = heads, a.d = d;
  a.per = rotate_each(n, heads, d);
  const int parts = div_up(heads, a.per);
  a.by_units = ig_fast_div(d / 16), a.by_parts = ig_fast_div(parts);
  a.total = n * parts * (d / 16);
  a.r = ig_rotary_refs(rotary, inverse);
  const dim3 grid((unsigned)div_up(a.total, 256)), block(256);
#define ROTATE(T, KIND)                                                                              \
  {                                                                                                  \
    auto k = rotate_rows<T, KIND>;                                                                   \
    IG_LAUNCH(ctx, IG_K_BUILD, k, grid, block, s, a);                                                \
  }
#define ROTATE_KIND(T)                                                                               \
  {                                                                                                  \
    if (a.r.kind == TURN_HALVES) ROTATE(T, TURN_HALVES)                                              \
    else if (a.r.kind == TURN_ADJACENT) ROTATE(T, TURN_ADJACENT)                                     \
    else if (a.r.kind == TURN_HALVES_4) ROTATE(T, TURN_HALVES_4)                                     \
    else if (a.r.kind == TURN_HALVES_2) ROTATE(T, TURN_HALVES_2)                                     \
    else ROTATE(T, TURN_HALVES_1)                                                                    \
  }
  if (dtype == IG_F16) ROTATE_KIND(half_t) else ROTATE_KIND(float)
  return IG_OK;
}

#define BY_DIM(T, E4M3, DO)                                                                          \
  switch (d->d) {                                                                                    \
    case 32: DO(T, 32, E4M3) break;                                                                  \
    case 64: DO(T, 64, E4M3) break;                                                                  \
    case 128: DO(T, 128, E4M3) break;                                                                \
    default: DO(T, 256, E4M3) break;                                                                 \
  }
#define BY_TYPE(DO)                                                                                  \
  {                                                                                                  \
    if (d->dtype == IG_F16 && p->code == IG_CODE_I8) BY_DIM(half_t, false, DO)                       \
    else if (d->dtype == IG_F16) BY_DIM(half_t, true, DO)                                            \
    else if (p->code == IG_CODE_I8) BY_DIM(float, false, DO)                                         \
    else BY_DIM(float, true, DO)                                                                     \
  }

int ig_launch_append_pages(ig_ctx *ctx, const ig_desc *d, const ig_pages *p, const ig_rotary *rotary, int Hq, int n_rows, const void *q,
                           const void *k, const void *v, long row_stride, const int32_t *n_append, const int32_t *kv_len, const int32_t *pos,
                           void *q_out, hipStream_t s) {
  AppendArgs a = {};
  a.p = ig_page_refs(d, p);
  a.q = q, a.k = k, a.v = v, a.q_out = q_out, a.n_append = n_append, a.kv_len = kv_len, a.pos = pos;
  a.q_stride = row_stride ? row_stride : (long)Hq * d->d, a.kv_stride = row_stride ? row_stride : (long)d->H * d->d;
  a.H = d->H, a.Hq = Hq, a.d = d->d, a.unit_shift = __builtin_ctz(d->d / 16), a.N = d->N, a.N_cap = d->N_cap, a.n_rows = n_rows;
  const AppendGrid g = append_grid(d, p, Hq, n_rows);
  a.per = g.per, a.q_per = g.q_per, a.kv_blocks = (int)g.kv_blocks, a.q_total = (int)g.q_total;
  a.by_pages = ig_fast_div(g.pages), a.by_parts = ig_fast_div(g.parts), a.by_rows = ig_fast_div(n_rows), a.by_q_parts = ig_fast_div(g.q_parts);
  a.r = ig_rotary_refs(rotary, 0);
  const dim3 grid((unsigned)(a.kv_blocks + div_up(a.q_total, g.team))), block(g.team);
#define APPEND(T, E4M3, KIND)                                                                        \
  {                                                                                                  \
    auto kernel = append_pages<T, E4M3, KIND>;                                                       \
    IG_LAUNCH(ctx, IG_K_BUILD, kernel, grid, block, s, a);                                           \
  }
#define APPEND_KIND(T, E4M3)                                                                         \
  {                                                                                                  \
    if (a.r.kind == TURN_NONE) APPEND(T, E4M3, TURN_NONE)                                            \
    else if (a.r.kind == TURN_HALVES) APPEND(T, E4M3, TURN_HALVES)                                   \
    else if (a.r.kind == TURN_ADJACENT) APPEND(T, E4M3, TURN_ADJACENT)                               \
    else if (a.r.kind == TURN_HALVES_4) APPEND(T, E4M3, TURN_HALVES_4)                               \
    else if (a.r.kind == TURN_HALVES_2) APPEND(T, E4M3, TURN_HALVES_2)                               \
    else APPEND(T, E4M3, TURN_HALVES_1)                                                              \
  }
#define APPEND_CODE(T)                                                                               \
  {                                                                                                  \
    if (p->code == IG_CODE_I8) APPEND_KIND(T, false) else APPEND_KIND(T, true)                       \
  }
  if (d->dtype == IG_F16) APPEND_CODE(half_t) else APPEND_CODE(float)
  return IG_OK;
}

static int gather_chunks(const ig_desc *d, int sel_stride) {
  return div_up((long)sel_stride * d->d * ig_elem_bytes(d->dtype), 256 * 16 * GATHER_ROWS);
}
long ig_gather_pages_threads(const ig_desc *d, int sel_stride) { return (long)d->B * d->H * gather_chunks(d, sel_stride) * 256; }

int ig_launch_gather_pages(ig_ctx *ctx, const ig_desc *d, const ig_pages *p, const int32_t *sel_idx, int sel_stride, const int32_t *sel_cnt,
                           void *K_sel, void *V_sel, hipStream_t s) {
  GatherArgs a = {};
  a.p = ig_page_refs(d, p);
  a.sel_idx = sel_idx, a.sel_cnt = sel_cnt, a.K_sel = K_sel, a.V_sel = V_sel, a.H = d->H, a.N_cap = d->N_cap, a.sel_stride = sel_stride;
  const int chunks = gather_chunks(d, sel_stride);
  a.by_chunks = ig_fast_div(chunks), a.by_H = ig_fast_div(d->H);
  const dim3 grid((unsigned)((long)d->B * d->H * chunks)), block(256);
#define GATHER(T, D, E4M3)                                                                           \
  {                                                                                                  \
    auto kernel = gather_pages<T, D, E4M3>;                                                          \
    IG_LAUNCH(ctx, IG_K_GATHER, kernel, grid, block, s, a);                                          \
  }
  BY_TYPE(GATHER)
  return IG_OK;
}
