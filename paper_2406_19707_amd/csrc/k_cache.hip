// Attention over a whole key / value pool: a prompt, a chunk of one or a single token with the accumulated
// attention weight of every slot, and a tree of drafted tokens over the pool (Section 2.1, softmax(q K^T) V;
// Section 2.3: the weights of earlier steps are what the eviction-based baselines rank a cache by).
#include "cache_device.h"

namespace {

// ---- few query rows, many cached rows ----------------------------------------------------------------
// The R = n_q * group query rows that share a pool (b,h) are taken 16 NT at a time; the cached rows of a slice
// are dealt to the four waves of a workgroup in tiles of 32 (float32: 16), and every wave keeps its own running
// maximum, sum and output for all 16 NT rows until the waves' states are joined through LDS.
//
// S^T = K Q^T and O^T = V^T P^T, both on 16x16 matrix instructions, so that a query row is a column, i.e. one
// lane of each group of 16: its maximum and sum need two exchanges a tile, and a factor of its own is one
// register.  Nothing of K or V passes through LDS:
//  - row i of the 16-row block a of S^T is the tile's token 8 (i/4) + 4 a + i%4, so that lane group g ends up
//    with the logits of the tokens 8g .. 8g+7, which are the eight k-entries it has to supply to P^T.
//  - a lane loads the same CJ = d/16 channels of those eight V rows (a wave-wide load is four whole rows), and
//    one byte permute each makes from them the pairs of tokens that V^T wants; row i of the output's block j is
//    the channel CJ i + j.
template <typename T, int D, int NT, bool TREE, bool LOGITS>
__global__ __launch_bounds__(256) void attend_stream(StreamArgs a) {
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int TT = HALF ? 32 : 16, MT = TT / 16, CJ = D / 16, RB = 16 * NT;
  constexpr int KCH = D * (int)sizeof(T) / 64;            // 16-byte pieces of a row that a lane holds
  constexpr int VT = HALF ? 8 : 4;                        // tokens of a tile that a lane group supplies
  constexpr int VW = CJ * (int)sizeof(T) / 4;             // words of a V row that a lane holds
  __shared__ __attribute__((aligned(16))) float box[RB * D];
  __shared__ float box_m[4][RB], box_l[4][RB];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;

  int work = xcd_order(blockIdx.x, a.per_xcd);
  if (work >= a.total) return;
  const int bh = a.by_pair.div(work);
  work -= bh * (int)a.by_pair.d;
  const int rb = a.nrb - 1 - a.by_slices.div(work);       // (a prompt's last rows see most: first)
  const int slice = a.by_slices.mod(work);
  const int b = a.by_H.div(bh), h = bh - b * (int)a.by_H.d;
  const int kv = length_of(a.kv_len, b, a.N, a.N_cap), nq = length_of(a.q_len, b, a.n_q, a.n_q);

  // what every row sees: slots below lim (and, in a tree, the nodes of its mask)
  int lim[NT];
  unsigned long long sees[NT];
  bool live[NT];
  const T *q = static_cast<const T *>(a.q);
  uint4 qf[NT][KCH];
  int lim_min = 0x7fffffff, lim_max = 0;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = rb * RB + n * 16 + i, iq = a.by_group.div(row), gq = row - iq * (int)a.by_group.d;
    live[n] = row < a.R && iq < nq;
    lim[n] = live[n] ? (TREE ? kv : max(0, kv - nq + iq + 1)) : 0x7fffffff;
    sees[n] = TREE && live[n] ? a.visible[(long)b * a.n_q + iq] & low_bits(nq) : 0;
    lim_min = min(lim_min, lim[n]);
    lim_max = max(lim_max, live[n] ? lim[n] : 0);
    const uint4 *src = reinterpret_cast<const uint4 *>(
        q + (((long)b * a.n_q + min(iq, a.n_q - 1)) * a.Hq + h * (int)a.by_group.d + gq) * D);
#pragma unroll
    for (int c = 0; c < KCH; ++c) qf[n][c] = flip_sign<T>(src[c * 4 + g], a.flip);
  }
  lim_min = wave_min_int(lim_min);
  lim_max = wave_max_int(lim_max);

  const int cache_tiles = (min(lim_max, kv) + TT - 1) / TT;
  const int tiles = cache_tiles + (TREE ? (nq + TT - 1) / TT : 0);
  const int per = (tiles + a.slices - 1) / a.slices;
  const int t_begin = min(tiles, slice * per), t_end = min(tiles, t_begin + per);

  const T *Kc = static_cast<const T *>(a.K) + (long)bh * a.N_cap * D, *Vc = static_cast<const T *>(a.V) + (long)bh * a.N_cap * D;
  uint4 k[MT][KCH];
  unsigned v[VT][VW];
  // (tokens past the end are read from the last one: what they hold is never used, and is finite if that is)
  auto load_k = [&](int tile) {
    const bool drafted = TREE && tile >= cache_tiles;
    const T *base = drafted ? static_cast<const T *>(a.k_tree) + ((long)b * a.n_q * a.by_H.d + h) * D : Kc;
    const long stride = drafted ? (long)a.by_H.d * D : D;
    const int t0 = (drafted ? tile - cache_tiles : tile) * TT, last = (drafted ? nq : kv) - 1;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int t = min(t0 + (HALF ? 8 * (i >> 2) + 4 * m + (i & 3) : i), last);
      const uint4 *src = reinterpret_cast<const uint4 *>(base + t * stride);
#pragma unroll
      for (int c = 0; c < KCH; ++c) k[m][c] = src[c * 4 + g];
    }
  };
  auto load_v = [&](int tile) {
    const bool drafted = TREE && tile >= cache_tiles;
    const T *base = drafted ? static_cast<const T *>(a.v_tree) + ((long)b * a.n_q * a.by_H.d + h) * D : Vc;
    const long stride = drafted ? (long)a.by_H.d * D : D;
    const int t0 = (drafted ? tile - cache_tiles : tile) * TT, last = (drafted ? nq : kv) - 1;
#pragma unroll
    for (int u = 0; u < VT; ++u)
      load_words<VW>(base + min(t0 + VT * g + u, last) * stride + CJ * i, v[u]);
  };

  floatx4 acc[NT][CJ];
  float m_run[NT], l_run[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int j = 0; j < CJ; ++j) acc[n][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  int tile = t_begin + w;
  if (tile < t_end) {
    load_k(tile);
    load_v(tile);
  }
  for (; tile < t_end; tile += 4) {
    const bool more = tile + 4 < t_end;
    floatx4 s[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m) s[n][m] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KCH; ++c)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n][m] = dot_step<T>(k[m][c], qf[n][c], s[n][m]);
    if (more) load_k(tile + 4);

    // masks, only where a tile holds something that some row does not see
    const bool drafted = TREE && tile >= cache_tiles;
    const int t0 = (drafted ? tile - cache_tiles : tile) * TT + VT * g;
    if (drafted) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!(t0 + 4 * m + r < 64 && (sees[n] >> ((t0 + 4 * m + r) & 63) & 1))) s[n][m][r] = -INFINITY;
    } else if ((tile + 1) * TT > lim_min) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (t0 + 4 * m + r >= lim[n]) s[n][m][r] = -INFINITY;
    }
    if (LOGITS) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (live[n]) {
          float *to = a.logits + ((long)bh * a.R + rb * RB + n * 16 + i) * a.logits_ld + t0;
#pragma unroll
          for (int m = 0; m < MT; ++m) *reinterpret_cast<floatx4 *>(to + 4 * m) = s[n][m];
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float top = s[n][0][0];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[n][m][r]);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float m_new = fmaxf(m_run[n], top);
      const float ref = m_new == -INFINITY ? 0.f : m_new * a.c;      // (nothing seen yet: every weight is exp2(-inf))
      if (__any(m_new > m_run[n])) {
        const float shrink = exp2_fast(m_run[n] * a.c - ref);
        l_run[n] *= shrink;
#pragma unroll
        for (int j = 0; j < CJ; ++j) acc[n][j] *= shrink;
        m_run[n] = m_new;
      }
      float sum = 0.f;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[n][m][r] = exp2_fast(fmaf(s[n][m][r], a.c, -ref));
          sum += s[n][m][r];
        }
      l_run[n] += sum;
    }
    if constexpr (HALF) {
      half8 p[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[n][e] = (half_t)s[n][e / 4][e % 4];
#pragma unroll
      for (int j = 0; j < CJ; ++j) {
        const half8 vt = column_of(v, j);
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, p[n], acc[n][j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < CJ; ++j)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[r][j]), s[n][0][r], acc[n][j], 0, 0, 0);
    }
    if (more) load_v(tile + 4);
  }

  // ---- the four waves' states joined: wave 0 ends up with that of the workgroup ----
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l_run[n] += __shfl_xor(l_run[n], 16, 64);
    l_run[n] += __shfl_xor(l_run[n], 32, 64);
    if (g == 0) {
      box_m[w][n * 16 + i] = m_run[n];
      box_l[w][n * 16 + i] = l_run[n];
    }
  }
  __syncthreads();
  float m_all[NT], l_all[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int at = n * 16 + i;
    const float m = fmaxf(fmaxf(box_m[0][at], box_m[1][at]), fmaxf(box_m[2][at], box_m[3][at]));
    const float ref = m == -INFINITY ? 0.f : m * a.c;
    m_all[n] = m;
    l_all[n] = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) l_all[n] += box_l[x][at] * exp2_fast(box_m[x][at] * a.c - ref);
    const float shrink = exp2_fast(m_run[n] * a.c - ref);
#pragma unroll
    for (int j = 0; j < CJ; ++j) acc[n][j] *= shrink;
  }
  for (int x = 3; x >= 1; --x) {
    if (w == x) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < CJ; ++j) *reinterpret_cast<floatx4 *>(box + ((n * CJ + j) * 64 + lane) * 4) = acc[n][j];
    }
    __syncthreads();
    if (w == 0) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < CJ; ++j) acc[n][j] += *reinterpret_cast<const floatx4 *>(box + ((n * CJ + j) * 64 + lane) * 4);
    }
    __syncthreads();
  }
  if (w) return;

  // ---- rows out: finished ones to `out`, the states of a slice to the workspace ----
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = rb * RB + n * 16 + i;
    if (!live[n]) continue;
    const float inv = l_all[n] > 0.f || l_all[n] != l_all[n] ? 1.f / l_all[n] : 0.f;
    if (a.slices == 1) {
      const int iq = a.by_group.div(row), gq = row - iq * (int)a.by_group.d;
      T *to = static_cast<T *>(a.out) + (((long)b * a.n_q + iq) * a.Hq + h * (int)a.by_group.d + gq) * D;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        T o[CJ];
#pragma unroll
        for (int j = 0; j < CJ; ++j) o[j] = (T)(acc[n][j][r] * inv);
        store_words<VW>(to + (4 * g + r) * CJ, o);
      }
      if (g == 0 && a.stats) a.stats[(long)bh * a.R + row] = make_float2(m_all[n], inv);
    } else {
      const long at = ((long)bh * a.slices + slice) * a.R + row;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < CJ; ++j) a.part[at * D + (4 * g + r) * CJ + j] = acc[n][j][r];
      if (g == 0) a.part_ml[at] = make_float2(m_all[n], l_all[n]);
    }
  }
}

// ---- joining the slices, and the weights of single-token calls ------------------------------------------
// A workgroup takes rows x, x + chunks, .. of a pool's R and, where logits were kept, the slots
// 1024 x .. of that pool: mass[t] += sum over the rows of exp2(c s - c m) / l.
template <typename T, bool LOGITS>
__global__ __launch_bounds__(256) void attend_join(StreamArgs a, float *mass, int D, FastDiv by_chunks) {
  __shared__ float2 stat[64];                              // (LOGITS: R <= 64)
  const int bh = by_chunks.div(blockIdx.x), x = by_chunks.mod(blockIdx.x), b = a.by_H.div(bh), h = bh - b * (int)a.by_H.d, tid = threadIdx.x;
  const int kv = length_of(a.kv_len, b, a.N, a.N_cap), nq = length_of(a.q_len, b, a.n_q, a.n_q);
  const int G = (int)a.by_group.d;
  auto joined = [&](int row, float *shrink_of) {           // the row's maximum and sum over all slices
    float m = -INFINITY, l = 0.f;
    for (int s = 0; s < a.slices; ++s) m = fmaxf(m, a.part_ml[((long)bh * a.slices + s) * a.R + row].x);
    const float ref = m == -INFINITY ? 0.f : m * a.c;
    for (int s = 0; s < a.slices; ++s) {
      const float2 ml = a.part_ml[((long)bh * a.slices + s) * a.R + row];
      l += ml.y * exp2_fast(ml.x * a.c - ref);
    }
    *shrink_of = ref;
    return make_float2(m, l > 0.f || l != l ? 1.f / l : 0.f);
  };
  if (a.slices > 1) {
    const int per = 256 / D < 1 ? 1 : 256 / D;             // rows a workgroup takes at a time
    for (int row = x * per + tid / D; row < nq * G && tid < per * D; row += (int)by_chunks.d * per) {
      float ref;
      const float2 st = joined(row, &ref);
      const int e = tid % D;
      float o = 0.f;
      for (int s = 0; s < a.slices; ++s) {
        const long at = ((long)bh * a.slices + s) * a.R + row;
        o += a.part[at * D + e] * exp2_fast(a.part_ml[at].x * a.c - ref);
      }
      const int iq = a.by_group.div(row), gq = row - iq * G;
      static_cast<T *>(a.out)[(((long)b * a.n_q + iq) * a.Hq + h * G + gq) * D + e] = (T)(o * st.y);
      if (a.stats && e == 0) a.stats[(long)bh * a.R + row] = st;
    }
  }
  if (LOGITS) {
    if (tid < a.R) {
      float ref;
      stat[tid] = a.slices > 1 ? joined(tid, &ref) : a.stats[(long)bh * a.R + tid];
    }
    __syncthreads();
    if (nq < 1) return;
    for (int t = x * 1024 + tid; t < min(kv, x * 1024 + 1024); t += 256) {
      float sum = 0.f;
      for (int row = 0; row < a.R; ++row) {
        const float ref = stat[row].x == -INFINITY ? 0.f : stat[row].x * a.c;
        sum = fmaf(exp2_fast(fmaf(a.logits[((long)bh * a.R + row) * a.logits_ld + t], a.c, -ref)), stat[row].y, sum);
      }
      mass[(long)bh * a.N_cap + t] += sum;
    }
  }
}

// ---- the weights of many query rows ------------------------------------------------------------------
// A wave keeps 32 (float32: 16) cached keys as the rows of S^T = K Q^T and takes every query row that sees
// them: mass[t] += sum over rows of exp2(c s - c m) / l, with the rows' final maxima and sums.
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_mass(StreamArgs a, float *mass, FastDiv by_chunks) {
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int TT = HALF ? 32 : 16, MT = TT / 16, KCH = D * (int)sizeof(T) / 64, VT = HALF ? 8 : 4;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int bh = by_chunks.div(blockIdx.x), x = by_chunks.mod(blockIdx.x);
  const int b = a.by_H.div(bh), h = bh - b * (int)a.by_H.d, G = (int)a.by_group.d;
  const int kv = length_of(a.kv_len, b, a.N, a.N_cap), nq = length_of(a.q_len, b, a.n_q, a.n_q);
  const int t0 = (x * 4 + w) * TT;
  if (t0 >= kv) return;
  const T *Kc = static_cast<const T *>(a.K) + (long)bh * a.N_cap * D;
  uint4 k[MT][KCH];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int t = min(t0 + (HALF ? 8 * (i >> 2) + 4 * m + (i & 3) : i), kv - 1);
#pragma unroll
    for (int c = 0; c < KCH; ++c) k[m][c] = reinterpret_cast<const uint4 *>(Kc + (long)t * D)[c * 4 + g];
  }
  float sum[MT][4] = {};
  // the first query that sees slot t0 is number t0 - (kv - nq)
  const int rows = nq * G, first = max(0, t0 - (kv - nq)) * G;
  for (int r0 = first; r0 < rows; r0 += 16) {
    const int row = min(r0 + i, rows - 1), iq = a.by_group.div(row), gq = row - iq * G;
    const bool live = r0 + i < rows;
    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const T *>(a.q) + (((long)b * a.n_q + iq) * a.Hq + h * G + gq) * D);
    const float2 st = a.stats[(long)bh * a.R + row];
    const float ref = st.x == -INFINITY ? 0.f : st.x * a.c, inv = live ? st.y : 0.f;
    const int lim = kv - nq + iq + 1;
    floatx4 s[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) s[m] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KCH; ++c) {
      const uint4 qf = flip_sign<T>(src[c * 4 + g], a.flip);
#pragma unroll
      for (int m = 0; m < MT; ++m) s[m] = dot_step<T>(k[m][c], qf, s[m]);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = exp2_fast(fmaf(s[m][r], a.c, -ref));
        sum[m][r] += live && t0 + VT * g + 4 * m + r < lim ? p * inv : 0.f;
      }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float all = row16_sum(sum[m][r]);
      const int t = t0 + VT * g + 4 * m + r;
      if (i == 0 && t < kv) mass[(long)bh * a.N_cap + t] += all;
    }
}

int div_up(long n, long d) { return (int)((n + d - 1) / d); }

// query rows a workgroup takes: 16, 32 or 64, what fits the registers beside the row's output
int row_block(const ig_desc *d, long R) {
  const int most = d->d > 128 ? 32 : 64;
  return R <= 16 ? 16 : (R <= 32 || most == 32 ? 32 : 64);
}

// Slices the cached rows of a pool are cut into: enough workgroups for about three a compute unit, while a
// wave of each still has a tile.
int slices_of(const ig_desc *d, long nrb, int n_keys) {
  const int tile = d->dtype == IG_F16 ? 32 : 16;
  const long want = (768 + d->B * (long)d->H * nrb - 1) / (d->B * (long)d->H * nrb);
  const long most = div_up(n_keys, 4 * tile);
  return (int)(want < 1 ? 1 : (want < most ? want : most) > 64 ? 64 : (want < most ? want : most));
}

}  // namespace

// Whether the logits of a call are kept for the weights (one query a sequence) instead of being worked out
// again from the keys.
static bool keeps_logits(const CacheCall &c) { return c.mass && c.n_q == 1 && c.group <= 64; }

CachePlan ig_cache_plan(const ig_desc *d, const CacheCall &c) {
  CachePlan p;
  const long R = (long)c.n_q * c.group, BH = (long)d->B * d->H;
  p.rb = row_block(d, R);
  p.nrb = div_up(R, p.rb);
  p.slices = slices_of(d, p.nrb, d->N + (c.k_tree ? c.n_q : 0));
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  p.logits_ld = ((long)d->N + 63) / 64 * 64;
  p.stats_at = take(c.mass ? BH * R * sizeof(float2) : 0);
  p.part_ml_at = take(p.slices > 1 ? BH * p.slices * R * sizeof(float2) : 0);
  p.part_at = take(p.slices > 1 ? BH * p.slices * R * d->d * sizeof(float) : 0);
  p.logits_at = take(keeps_logits(c) ? BH * R * p.logits_ld * sizeof(float) : 0);
  p.bytes = at;
  return p;
}

int ig_launch_cache(ig_ctx *ctx, const ig_desc *d, const CacheCall &c, const CachePlan &p, char *ws, hipStream_t stream) {
  const bool tree = c.k_tree != nullptr, logits = keeps_logits(c);
  const long BH = (long)d->B * d->H;
  StreamArgs a = {};
  a.q = c.q, a.K = c.K, a.V = c.V, a.k_tree = c.k_tree, a.v_tree = c.v_tree, a.out = c.out;
  a.visible = c.visible, a.q_len = c.q_len, a.kv_len = c.kv_len;
  a.n_q = c.n_q, a.R = c.n_q * c.group, a.Hq = d->H * c.group, a.N = d->N, a.N_cap = d->N_cap;
  a.nrb = p.nrb, a.slices = p.slices, a.total = (int)(BH * p.nrb * p.slices), a.per_xcd = div_up(a.total, 8);
  a.by_pair = ig_fast_div(p.nrb * p.slices), a.by_slices = ig_fast_div(p.slices);
  a.by_H = ig_fast_div(d->H), a.by_group = ig_fast_div(c.group);
  a.flip = d->scale < 0.f ? 1 : (d->scale == 0.f ? 2 : 0);
  a.c = (d->scale == 0.f ? 1.f : fabsf(d->scale)) * 1.44269504088896340736f;
  a.stats = c.mass ? reinterpret_cast<float2 *>(ws + p.stats_at) : nullptr;
  a.part_ml = reinterpret_cast<float2 *>(ws + p.part_ml_at);
  a.part = reinterpret_cast<float *>(ws + p.part_at);
  a.logits = reinterpret_cast<float *>(ws + p.logits_at);
  a.logits_ld = p.logits_ld;
  const dim3 grid(a.per_xcd * 8), block(256);
#define STREAM(T, D, NT)                                                                             \
  {                                                                                                  \
    if (tree) {                                                                                      \
      auto k = attend_stream<T, D, NT, true, false>;                                                 \
      IG_LAUNCH(ctx, IG_K_CACHE, k, grid, block, stream, a);                                         \
    } else if (logits) {                                                                             \
      auto k = attend_stream<T, D, NT, false, true>;                                                 \
      IG_LAUNCH(ctx, IG_K_CACHE, k, grid, block, stream, a);                                         \
    } else {                                                                                         \
      auto k = attend_stream<T, D, NT, false, false>;                                                \
      IG_LAUNCH(ctx, IG_K_CACHE, k, grid, block, stream, a);                                         \
    }                                                                                                \
  }
#define STREAM_ROWS(T, D)                                                                            \
  {                                                                                                  \
    if (p.rb == 16) STREAM(T, D, 1)                                                                  \
    else if (p.rb == 32) STREAM(T, D, 2)                                                             \
    else if constexpr (D <= 128) STREAM(T, D, 4)                                                     \
  }
#define BY_DIM(T, DO)                                                                                \
  switch (d->d) {                                                                                    \
    case 32: DO(T, 32) break;                                                                        \
    case 64: DO(T, 64) break;                                                                        \
    case 128: DO(T, 128) break;                                                                      \
    default: DO(T, 256) break;                                                                       \
  }
  if (d->dtype == IG_F16) {
    BY_DIM(half_t, STREAM_ROWS)
  } else {
    BY_DIM(float, STREAM_ROWS)
  }
  if (p.slices > 1 || logits) {
    const int chunks = logits ? div_up(d->N, 1024) : 1;
    const int rows = p.slices > 1 ? div_up((long)a.R * d->d, 256) : 1;
    const FastDiv by_chunks = ig_fast_div(chunks > rows ? chunks : rows);
    const dim3 jgrid((unsigned)(by_chunks.d * BH));
#define JOIN(T)                                                                                      \
  {                                                                                                  \
    if (logits) {                                                                                    \
      auto k = attend_join<T, true>;                                                                 \
      IG_LAUNCH(ctx, IG_K_CACHE, k, jgrid, block, stream, a, c.mass, (int)d->d, by_chunks);                     \
    } else {                                                                                         \
      auto k = attend_join<T, false>;                                                                \
      IG_LAUNCH(ctx, IG_K_CACHE, k, jgrid, block, stream, a, (float *)nullptr, (int)d->d, by_chunks);           \
    }                                                                                                \
  }
    if (d->dtype == IG_F16) JOIN(half_t) else JOIN(float)
  }
  if (c.mass && !logits) {
    const int tile = d->dtype == IG_F16 ? 32 : 16;
    const FastDiv by_chunks = ig_fast_div(div_up(d->N, 4 * tile));
    const dim3 mgrid((unsigned)(by_chunks.d * BH));
#define MASS(T, D)                                                                                   \
  {                                                                                                  \
    auto k = attend_mass<T, D>;                                                                      \
    IG_LAUNCH(ctx, IG_K_CACHE, k, mgrid, block, stream, a, c.mass, by_chunks);                                  \
  }
    if (d->dtype == IG_F16) {
      BY_DIM(half_t, MASS)
    } else {
      BY_DIM(float, MASS)
    }
  }
  return IG_OK;
}

// What ig_reserve_cache sizes the workspace for.  More rows mean fewer slices, so the largest need is not that of
// the largest call: every number of tokens is looked at for which the pools are still cut into slices.
size_t ig_cache_reserve_bytes(const ig_desc *d, int group, int n_q) {
  ig_desc full = *d;
  full.N = d->N_cap;
  const int half_keep = full.N / 2 < 1 ? 1 : full.N / 2;
  size_t most = ig_evict_workspace(&full, half_keep);
  static float weights;
  auto look = [&](int n) {
    CacheCall c = {};
    c.group = group, c.n_q = n, c.mass = &weights;
    const CachePlan p = ig_cache_plan(&full, c);
    if (p.bytes > most) most = p.bytes;
    if (n <= 64) {
      c.mass = nullptr, c.k_tree = &weights;
      const CachePlan t = ig_cache_plan(&full, c);
      if (t.bytes > most) most = t.bytes;
      return p.slices > 1 || t.slices > 1;
    }
    return p.slices > 1;
  };
  for (int n = 1; n <= n_q && look(n); ++n) {
  }
  look(n_q);
  return most;
}
