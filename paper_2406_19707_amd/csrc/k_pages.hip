// Rotary embedding of rows, their append to pages of 8-bit codes with a scale for each page and head, and rows read back.
#include "page_device.h"

namespace {

int div_up(long n, long d) { return (int)((n + d - 1) / d); }

// ---- rotation ------------------------------------------------------------------------------------------------------
// A thread takes one unit of a token, works out its eight turns once, and takes HEADS heads of it.
constexpr int ROTATE_HEADS = 8;
struct RotateArgs {
  const void *x;
  void *out;
  const int32_t *pos;
  long x_stride, out_stride;
  int n, heads, d, chunks;            // chunks of ROTATE_HEADS heads
  long total;                         // units of all tokens, times chunks
  FastDiv by_units, by_chunks;
  RotaryRefs r;
};
template <typename T>
__device__ __forceinline__ void rotate_heads(const T *x, T *out, int d, int h0, int heads, int s, int pos, const RotaryRefs &r) {
  float2 turn[8];
  turns_of(s, pos, r, turn);
  for (int h = h0; h < min(h0 + ROTATE_HEADS, heads); ++h) {
    Unit<T> u;
    u.load(x + (long)h * d, s, r.dims, r.kind);
    float v[16];
    u.get(v);
    rotate_unit(v, s, r.dims, r.kind, turn);
    Unit<T>::store(out + (long)h * d, s, r.dims, r.kind, v);
  }
}
template <typename T> __global__ __launch_bounds__(256) void rotate_rows(RotateArgs a) {
  const int u = blockIdx.x * 256 + threadIdx.x;
  if (u >= a.total) return;
  const int at = a.by_units.div(u), s = u - at * (int)a.by_units.d, i = a.by_chunks.div(at), chunk = at - i * a.chunks;
  rotate_heads<T>(static_cast<const T *>(a.x) + i * a.x_stride, static_cast<T *>(a.out) + i * a.out_stride, a.d, chunk * ROTATE_HEADS, a.heads, s,
                  a.pos[i], a.r);
}

// ---- append --------------------------------------------------------------------------------------------------------
// A workgroup takes the new rows of one page of a sequence, head after head of APPEND_HEADS, K and V together: two
// units of 16 channels a thread, their turns worked out once for all heads.  The largest value of a head's rows gives the scale.
constexpr int APPEND_HEADS = 8, APPEND_UNITS = 2;
struct AppendArgs {
  PageRefs p;
  const void *q, *k, *v;
  void *q_out;
  const int32_t *n_append, *kv_len, *pos;
  long q_stride, kv_stride;
  int B, H, Hq, N, N_cap, n_rows;
  int pages, chunks, q_chunks;        // pages a sequence's rows touch at most, chunks of heads
  int kv_blocks;                      // workgroups of the pages; those behind them rotate queries
  long q_total;
  FastDiv by_pages, by_chunks, by_rows, by_q_chunks, by_q_units;
  RotaryRefs r;
};
// the value to be stored: 0 for one that is not finite
__device__ __forceinline__ float finite_or_zero(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.f : x; }

template <typename T, int D, bool E4M3> __global__ void append_pages(AppendArgs a) {
  constexpr int UNITS = D / 16;
  __shared__ float tops[2][2][16];
  const int tid = threadIdx.x, team = blockDim.x;
  if ((int)blockIdx.x >= a.kv_blocks) {
    const int u = (blockIdx.x - a.kv_blocks) * team + tid;
    if (u >= a.q_total) return;
    const int at = u / UNITS, s = u % UNITS, i = a.by_q_chunks.div(at), chunk = at - i * a.q_chunks;
    const int b = a.by_rows.div(i), j = i - b * a.n_rows;
    if (j >= (a.n_append ? min(max(a.n_append[b], 0), a.n_rows) : a.n_rows)) return;
    const int first = a.pos ? a.pos[b] : (a.kv_len ? min(max(a.kv_len[b], 0), a.N_cap) : a.N);
    rotate_heads<T>(static_cast<const T *>(a.q) + i * a.q_stride, static_cast<T *>(a.q_out) + (long)i * a.Hq * D, D, chunk * ROTATE_HEADS, a.Hq, s,
                    first + j, a.r);
    return;
  }
  const int at = a.by_pages.div(blockIdx.x), p = blockIdx.x - at * a.pages, b = a.by_chunks.div(at), chunk = at - b * a.chunks;
  const int start = a.kv_len ? min(max(a.kv_len[b], 0), a.N_cap) : a.N;
  const int n = min(a.n_append ? min(max(a.n_append[b], 0), a.n_rows) : a.n_rows, a.N_cap - start);
  const int number = (start >> a.p.shift) + p, slot0 = number << a.p.shift;
  const int r0 = max(start, slot0), r1 = min(start + n, slot0 + (1 << a.p.shift));
  if (r0 >= r1) return;
  const int entry = a.p.table[(long)b * a.p.stride + number];
  if ((unsigned)entry >= a.p.n_pages) return;
  const int held = r0 - slot0, total = (r1 - r0) * UNITS, first_pos = (a.pos ? a.pos[b] : start) + (r0 - start);

  int row[APPEND_UNITS], unit[APPEND_UNITS];
  float2 turn[APPEND_UNITS][8];
  bool mine[APPEND_UNITS];
#pragma unroll
  for (int k = 0; k < APPEND_UNITS; ++k) {
    const int u = tid + k * team;
    mine[k] = u < total;
    row[k] = mine[k] ? u / UNITS : 0, unit[k] = u % UNITS;
    turns_of(unit[k], first_pos + row[k], a.r, turn[k]);
  }
  const int h_end = min((chunk + 1) * APPEND_HEADS, a.H);
  for (int h = chunk * APPEND_HEADS; h < h_end; ++h) {
    float x[2][APPEND_UNITS][16];                          // of K, of V
    float top[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < APPEND_UNITS; ++k) {
      // (a thread without a unit reads the first row and stores nothing)
      const long src = ((long)b * a.n_rows + (r0 - start) + row[k]) * a.kv_stride + (long)h * D;
      Unit<T> ku, vu;
      ku.load(static_cast<const T *>(a.k) + src, unit[k], a.r.dims, a.r.kind);
      vu.load(static_cast<const T *>(a.v) + src, unit[k], 0, TURN_NONE);
      ku.get(x[0][k]);
      vu.get(x[1][k]);
      rotate_unit(x[0][k], unit[k], a.r.dims, a.r.kind, turn[k]);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[kv][k][e] = finite_or_zero(x[kv][k][e]);
          if (mine[k]) top[kv] = fmaxf(top[kv], fabsf(x[kv][k][e]));
        }
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      top[kv] = wave_max(top[kv]);
      if (team > 64 && tid % 64 == 0) tops[h & 1][kv][tid / 64] = top[kv];
    }
    const long scale_at = (long)entry * a.H + h;
    float *scales[2] = {a.p.K_scale + scale_at, a.p.V_scale + scale_at};
    int before[2] = {SCALE_LEAST, SCALE_LEAST};
    if (held)
      for (int kv = 0; kv < 2; ++kv) before[kv] = scale_exponent(*scales[kv]);
    if (team > 64) {
      // (the scales are there before any thread may store a new one)
      asm volatile("" : "+v"(before[0]), "+v"(before[1]));
      __syncthreads();
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
        for (int w = 0; w < team / 64; ++w) top[kv] = fmaxf(top[kv], tops[h & 1][kv][w]);
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const int e2 = max(before[kv], exponent_for<E4M3>(top[kv]));
      char *page = (kv ? a.p.V : a.p.K) + (unsigned long)(unsigned)entry * a.p.page_bytes + ((long)h << a.p.shift) * D;
      if (held && e2 > before[kv]) {
        const float by = exp2_int(max(before[kv] - e2, -126));
        for (int u = tid; u < held * (D / 16); u += team) {
          uint4 *c = reinterpret_cast<uint4 *>(page) + u;
          uint4 v = *c;
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
        char *to = page + (long)(held + row[k]) * D;
        float *f = x[kv][k];
#pragma unroll
        for (int e = 0; e < 16; ++e) f[e] *= inv;
        unsigned c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = encode4<E4M3>(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
        if (kv == 0 && a.r.kind == TURN_ANY) {
#pragma unroll
          for (int e = 0; e < 16; ++e) to[any_channel(8 * unit[k] + e % 8, e / 8, a.r.dims)] = (char)(c[e / 4] >> e % 4 * 8);
        } else {
          const Runs at = runs_of(unit[k], a.r.dims, kv ? TURN_NONE : a.r.kind);
          *reinterpret_cast<uint2 *>(to + at.first) = make_uint2(c[0], c[1]);
          *reinterpret_cast<uint2 *>(to + at.second) = make_uint2(c[2], c[3]);
        }
      }
      if (tid == 0 && (!held || e2 > before[kv])) *scales[kv] = exp2_int(e2);
    }
  }
}

// ---- rows read back ------------------------------------------------------------------------------------------------
// A thread takes 16 channels of a listed row, of K and of V.
struct GatherArgs {
  PageRefs p;
  const int32_t *sel_idx, *sel_cnt;
  void *K_sel, *V_sel;
  int H, N_cap, sel_stride;
  FastDiv by_chunks, by_H;
};
template <typename T, int D, bool E4M3> __global__ __launch_bounds__(256) void gather_pages(GatherArgs a) {
  constexpr int UNITS = D / 16, ROWS = 256 / UNITS;
  const int bh = a.by_chunks.div(blockIdx.x), chunk = blockIdx.x - bh * (int)a.by_chunks.d, b = a.by_H.div(bh), h = bh - b * a.H;
  const int j = chunk * ROWS + threadIdx.x / UNITS, s = threadIdx.x % UNITS;
  if (j >= min(a.sel_cnt[bh], a.sel_stride)) return;
  const int slot = min(max(a.sel_idx[(long)bh * a.sel_stride + j], 0), a.N_cap - 1);
  const unsigned page = page_read(a.p, a.p.table[(long)b * a.p.stride + (slot >> a.p.shift)]);
  const unsigned long from = (unsigned long)page * a.p.page_bytes + (((unsigned long)h << a.p.shift) + (slot & ((1 << a.p.shift) - 1))) * D + s * 16;
  const uint4 codes[2] = {*reinterpret_cast<const uint4 *>(a.p.K + from), *reinterpret_cast<const uint4 *>(a.p.V + from)};
  const float scales[2] = {a.p.K_scale[(long)page * a.H + h], a.p.V_scale[(long)page * a.H + h]};
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const float by = exp2_int(scale_exponent(scales[kv]));
    const unsigned w[4] = {codes[kv].x, codes[kv].y, codes[kv].z, codes[kv].w};
    float x[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const floatx4 f = decode4<E4M3>(w[i]) * by;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = f[e];
    }
    T *to = static_cast<T *>(kv ? a.V_sel : a.K_sel) + ((long)bh * a.sel_stride + j) * D + s * 16;
    Run8<T>::store(to, x);
    Run8<T>::store(to + 8, x + 8);
  }
}

int head_chunks(int heads, int per) { return (heads + per - 1) / per; }
// Pages that n_rows new rows of a sequence touch at most, and threads of a workgroup: a page's new rows in two units each.
int append_page_count(const ig_pages *p, int n_rows) { return (n_rows + p->page_size - 2) / p->page_size + 1; }
int append_team(const ig_desc *d, const ig_pages *p, int n_rows) {
  const int units = (n_rows < p->page_size ? n_rows : p->page_size) * d->d / 16;
  int team = 64;
  while (team * APPEND_UNITS < units) team *= 2;
  return team;
}

}  // namespace

long ig_rotate_threads(int n, int heads, int d) { return ((long)n * head_chunks(heads, ROTATE_HEADS) * (d / 16) + 255) / 256 * 256; }

int ig_launch_rotate(ig_ctx *ctx, int dtype, int n, int heads, int d, const ig_rotary *rotary, int inverse, const int32_t *pos, const void *x,
                     long x_stride, void *out, long out_stride, hipStream_t s) {
  RotateArgs a = {};
  a.x = x, a.out = out, a.pos = pos, a.x_stride = x_stride, a.out_stride = out_stride, a.n = n, a.heads = heads, a.d = d;
  a.chunks = head_chunks(heads, ROTATE_HEADS), a.by_units = ig_fast_div(d / 16), a.by_chunks = ig_fast_div(a.chunks);
  a.total = (long)n * a.chunks * (d / 16);
  a.r = ig_rotary_refs(rotary, inverse);
  const dim3 grid((unsigned)div_up(a.total, 256)), block(256);
  if (dtype == IG_F16) {
    auto k = rotate_rows<half_t>;
    IG_LAUNCH(ctx, IG_K_BUILD, k, grid, block, s, a);
  } else {
    auto k = rotate_rows<float>;
    IG_LAUNCH(ctx, IG_K_BUILD, k, grid, block, s, a);
  }
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

long ig_append_pages_threads(const ig_desc *d, const ig_pages *p, int Hq, int n_rows) {
  const int team = append_team(d, p, n_rows);
  const long kv = (long)d->B * append_page_count(p, n_rows) * head_chunks(d->H, APPEND_HEADS) * team;
  return kv + ((long)d->B * n_rows * head_chunks(Hq, ROTATE_HEADS) * (d->d / 16) + team - 1) / team * team;
}

int ig_launch_append_pages(ig_ctx *ctx, const ig_desc *d, const ig_pages *p, const ig_rotary *rotary, int Hq, int n_rows, const void *q,
                           const void *k, const void *v, long row_stride, const int32_t *n_append, const int32_t *kv_len, const int32_t *pos,
                           void *q_out, hipStream_t s) {
  AppendArgs a = {};
  a.p = ig_page_refs(d, p);
  a.q = q, a.k = k, a.v = v, a.q_out = q_out, a.n_append = n_append, a.kv_len = kv_len, a.pos = pos;
  a.q_stride = row_stride ? row_stride : (long)Hq * d->d, a.kv_stride = row_stride ? row_stride : (long)d->H * d->d;
  a.B = d->B, a.H = d->H, a.Hq = Hq, a.N = d->N, a.N_cap = d->N_cap, a.n_rows = n_rows;
  a.pages = append_page_count(p, n_rows), a.chunks = head_chunks(d->H, APPEND_HEADS), a.q_chunks = head_chunks(Hq, ROTATE_HEADS);
  a.kv_blocks = d->B * a.pages * a.chunks;
  a.q_total = q ? (long)d->B * n_rows * a.q_chunks * (d->d / 16) : 0;
  a.by_pages = ig_fast_div(a.pages), a.by_chunks = ig_fast_div(a.chunks), a.by_rows = ig_fast_div(n_rows);
  a.by_q_chunks = ig_fast_div(a.q_chunks > 0 ? a.q_chunks : 1), a.by_q_units = ig_fast_div(d->d / 16);
  a.r = ig_rotary_refs(rotary, 0);
  const int team = append_team(d, p, n_rows);
  const dim3 grid((unsigned)(a.kv_blocks + div_up(a.q_total, team))), block(team);
#define APPEND(T, D, E4M3)                                                                           \
  {                                                                                                  \
    auto kernel = append_pages<T, D, E4M3>;                                                          \
    IG_LAUNCH(ctx, IG_K_BUILD, kernel, grid, block, s, a);                                           \
  }
  BY_TYPE(APPEND)
  return IG_OK;
}

long ig_gather_pages_threads(const ig_desc *d, int sel_stride) {
  return (long)d->B * d->H * div_up((long)sel_stride * (d->d / 16), 256) * 256;
}

int ig_launch_gather_pages(ig_ctx *ctx, const ig_desc *d, const ig_pages *p, const int32_t *sel_idx, int sel_stride, const int32_t *sel_cnt,
                           void *K_sel, void *V_sel, hipStream_t s) {
  GatherArgs a = {};
  a.p = ig_page_refs(d, p);
  a.sel_idx = sel_idx, a.sel_cnt = sel_cnt, a.K_sel = K_sel, a.V_sel = V_sel, a.H = d->H, a.N_cap = d->N_cap, a.sel_stride = sel_stride;
  const int chunks = div_up((long)sel_stride * (d->d / 16), 256);
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
