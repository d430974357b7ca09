// Eviction of a pool's slots by accumulated attention weight (Section 5.3: the cache of a fixed budget that the
// rehearsal is compared with), and the append of several rows to ragged sequences.
#include <type_traits>

#include "cache_device.h"

namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// order-preserving image of a weight: larger <-> larger unsigned, -0 as +0, NaN below everything; between 1 and +inf's
// 0xff800000, so that 0 and ~0u are left for slots that are ranked without their weight
__device__ __forceinline__ unsigned weight_key(float s) {
  const unsigned b = __float_as_uint(s + 0.0f);
  return s != s ? 1u : ((b & 0x80000000u) ? ~b : (b | 0x80000000u));
}

struct EvictArgs {
  const int32_t *kv_len, *protect_from, *idx;
  float *mass;
  int32_t *born;
  void *K, *V, *slab;
  int32_t *count, *moves;          // [B*H]; [B*H][2][most]: slots that move, slots they fill
  int H, N, N_cap, keep, most, units, d, r, nTiles;
  FastDiv by_H, by_units, by_chunks;
};

// rows j0 .. j1-1 of a pool's list of moves: K and V rows in 16-byte units, then the slab's channels
template <typename T, int THREADS>
__device__ __forceinline__ void move_rows(const EvictArgs &a, int bh, const int32_t *from, const int32_t *to, int j0, int j1) {
  constexpr int TILE = IG_WAVE * SlabElem<T>::TPL, BATCH = 4;
  u32x4 *K = static_cast<u32x4 *>(a.K) + (long)bh * a.N_cap * a.units, *V = static_cast<u32x4 *>(a.V) + (long)bh * a.N_cap * a.units;
  const int total = (j1 - j0) * a.units;
  for (int u0 = threadIdx.x; u0 < total; u0 += THREADS * BATCH) {
    u32x4 kv[BATCH], vv[BATCH];
    int at[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int u = min(u0 + THREADS * i, total - 1), j = a.by_units.div(u), c = u - j * a.units;
      const long s = (long)from[j0 + j] * a.units + c;
      at[i] = to[j0 + j];
      kv[i] = K[s];
      vv[i] = V[s];
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int u = u0 + THREADS * i;
      if (u < total) {
        const long s = (long)at[i] * a.units + a.by_units.mod(u);
        K[s] = kv[i];
        V[s] = vv[i];
      }
    }
  }
  if (a.slab) {
    const int h = a.by_H.mod(bh);
    T *slab = static_cast<T *>(a.slab) + (long)bh * a.nTiles * a.r * TILE;
    const T *Krows = static_cast<const T *>(a.K) + (long)bh * a.N_cap * a.d;
    const int rows = j1 - j0;
    for (int c = threadIdx.x / 16; c < a.r; c += THREADS / 16) {
      const int col = min(max(a.idx[h * a.r + c], 0), a.d - 1);
      for (int j = threadIdx.x % 16; j < rows; j += 16) {
        const int s = to[j0 + j];
        // (slots that move are not written by the move, so their rows still hold what went to slot s)
        slab[((long)(s / TILE) * a.r + c) * TILE + s % TILE] = Krows[(long)from[j0 + j] * a.d + col];
      }
    }
  }
}

// One workgroup per pool.  The keep-th largest key by radix selection (keys in registers, KPT of them a thread,
// or read again in every pass), then two ordered lists: slots from `keep` on that stay, slots below it that do
// not.  They are equally long, and the j-th of the one fills the j-th of the other: no row is both read and
// written, so the rows move in place and in any order.  Bound by its steps in turn (loads, three passes over the keys
// with a barrier each, two ordered counts): 512 pools of 4096 slots 14.7 us.  512 threads while eight keys each hold a
// pool; 1024 with 32 each up to 32768 slots, beyond that the keys are read again in every pass.
template <typename T, int THREADS, int KPT, bool MOVE>
__global__ __launch_bounds__(THREADS) void evict_select(EvictArgs a) {
  constexpr int NW = THREADS / 64, U = KPT > 0 ? KPT : 8;
  __shared__ __attribute__((aligned(16))) unsigned hist[3][RADIX_WORDS];
  __shared__ int w_safe[NW], w_eq[NW], w_src[NW], w_dst[NW];
  const int bh = blockIdx.x, b = a.by_H.div(bh), tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = length_of(a.kv_len, b, a.N, a.N_cap);
  if (n <= a.keep) {
    if (tid == 0 && !MOVE) a.count[bh] = 0;
    return;
  }
  float *mass = a.mass + (long)bh * a.N_cap;
  int32_t *born = a.born ? a.born + (long)bh * a.N_cap : nullptr;
  const int guard = a.protect_from ? a.protect_from[b] : 0;
  const int chunk = KPT > 0 ? KPT * 64 : ((n + THREADS - 1) / THREADS) * 64;
  const int t0 = min(n, w * chunk), t1 = min(n, t0 + chunk);
  unsigned key[U];
  // (protected slots rank before all others; where there are more of them than may stay, they alone are ranked)
  bool crowded = false;
  unsigned apart = ~0u;                                   // the key of slots that are decided without their weight
  auto load = [&](int t, auto together) {                 // so many at a time
    constexpr int P = decltype(together)::value;
#pragma unroll
    for (int i0 = 0; i0 < U; i0 += P) {
      float m[P];
      int age[P];
      if (P < U) t = (int)opaque(t);                      // (not all addresses ahead)
#pragma unroll
      for (int i = 0; i < P; ++i) m[i] = mass[min(t + (i0 + i) * 64 + lane, n - 1)];
      if (a.protect_from) {
#pragma unroll
        for (int i = 0; i < P; ++i) age[i] = born[min(t + (i0 + i) * 64 + lane, n - 1)];
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const bool safe = a.protect_from && age[i] >= guard;
        key[i0 + i] = safe == crowded ? weight_key(m[i]) : apart;
        if (P < U) keep_here(key[i0 + i]);
      }
    }
  };
  typedef std::integral_constant<int, U> all_of_them;
  // f(slot, its key, whether there is such a slot) in order of the slots, 64 a call
  auto each = [&](auto &&f) {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int i = 0; i < U; ++i) f(t0 + i * 64 + lane, key[i], t0 + i * 64 + lane < t1);
    } else {
      for (int t = t0; t < t1; t += U * 64) {
        load(t, all_of_them());
#pragma unroll
        for (int i = 0; i < U; ++i) f(t + i * 64 + lane, key[i], t + i * 64 + lane < t1);
      }
    }
  };
  if constexpr (KPT > 0) load(t0, all_of_them());
  for (int i = tid; i < 3 * RADIX_WORDS / 4; i += THREADS) reinterpret_cast<uint4 *>(&hist[0][0])[i] = make_uint4(0, 0, 0, 0);
  // The protected slots, which all have one key, are counted by ballots and left out of the histograms, where whole
  // waves of them would add to one word.
  int safe = 0;
  each([&](int, unsigned k, bool there) { safe += __popcll(__ballot(there && k == ~0u)); });
  if (lane == 0) w_safe[w] = safe;
  __syncthreads();
  safe = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) safe += w_safe[i];

  // slots with a key above lim stay, and the first `need` of those equal to it
  unsigned lim = 0;
  int need = a.keep - safe;
  if (need == 0) {                                        // (the protected slots, all of them, and no others)
    lim = ~0u;
    need = a.keep;
  } else if (need < 0) {
    crowded = true;
    apart = 0;
    need = a.keep;
    // (four at a time: all together need registers that the other path has not)
    if constexpr (KPT > 0) load(t0, std::integral_constant<int, 4>());
  }
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    if (lim == ~0u && pass == 0) break;
    each([&](int, unsigned k, bool there) {
      if (there && k != apart) radix_add(hist[pass], pass, k, lim);
    });
    __syncthreads();
    bool whole;
    lim |= radix_digit(hist[pass], lane, need, &whole) << radix_shift(pass);
    if (pass < 2 && whole && lim > 0) {
      lim -= 1;
      need = 0;
      break;
    }
  }
  int eq = 0;
  each([&](int, unsigned k, bool there) { eq += __popcll(__ballot(there && k == lim)); });
  if (lane == 0) w_eq[w] = eq;
  __syncthreads();
  int eq_first = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) eq_first += i < w ? w_eq[i] : 0;
  int src = 0, dst = 0, eq_rank = eq_first;
  auto stays = [&](unsigned k, bool there) {
    const unsigned long long be = __ballot(there && k == lim);
    const bool s = there && (k > lim || (k == lim && eq_rank + lanes_below(be) < need));
    eq_rank += __popcll(be);
    return s;
  };
  each([&](int t, unsigned k, bool there) {
    const bool s = stays(k, there);
    src += __popcll(__ballot(s && t >= a.keep));
    dst += __popcll(__ballot(there && !s && t < a.keep));
  });
  if (lane == 0) {
    w_src[w] = src;
    w_dst[w] = dst;
  }
  __syncthreads();
  int total = 0, src_at = 0, dst_at = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    src_at += i < w ? w_src[i] : 0;
    dst_at += i < w ? w_dst[i] : 0;
    total += w_src[i];
  }
  int32_t *from = a.moves + (long)bh * 2 * a.most, *to = from + a.most;
  eq_rank = eq_first;
  each([&](int t, unsigned k, bool there) {
    const bool s = stays(k, there);
    const bool moves = s && t >= a.keep, hole = there && !s && t < a.keep;
    const unsigned long long bs = __ballot(moves), bd = __ballot(hole);
    if (moves) from[src_at + lanes_below(bs)] = t;
    if (hole) to[dst_at + lanes_below(bd)] = t;
    src_at += __popcll(bs);
    dst_at += __popcll(bd);
  });
  if (!MOVE && tid == 0) a.count[bh] = total;
  __syncthreads();
  for (int j = tid; j < total; j += THREADS) {
    const int s = from[j], t = to[j];
    mass[t] = mass[s];
    if (born) born[t] = born[s];
  }
  if constexpr (MOVE) move_rows<T, THREADS>(a, bh, from, to, 0, total);
}

// The eviction of a decode step, one slot too many (N = keep + 1): the slot that ranks last makes room for the last
// slot.  Bound by the trips through memory: the last slot's rows, weight and
// position are asked for with the weights.  256 pools of 2049 slots: 5.2 us, 10.1 with the radix selection.
template <typename T, int THREADS> __global__ __launch_bounds__(THREADS) void evict_one(EvictArgs a) {
  constexpr int NW = THREADS / 64, U = 8, TILE = IG_WAVE * SlabElem<T>::TPL;
  __shared__ unsigned long long w_best[NW];
  const int bh = blockIdx.x, b = a.by_H.div(bh), tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = length_of(a.kv_len, b, a.N, a.N_cap), last = a.keep;
  float *mass = a.mass + (long)bh * a.N_cap;
  int32_t *born = a.born ? a.born + (long)bh * a.N_cap : nullptr;
  const int guard = a.protect_from ? a.protect_from[b] : 0;
  u32x4 *K = static_cast<u32x4 *>(a.K) + (long)bh * a.N_cap * a.units, *V = static_cast<u32x4 *>(a.V) + (long)bh * a.N_cap * a.units;
  const bool copies = tid < a.units;               // (the host: a row has at most 256 units)
  u32x4 kv = {}, vv = {};
  if (copies) {                                    // (slot `keep` is inside the pool: N_cap >= N > keep)
    kv = K[(long)last * a.units + tid];
    vv = V[(long)last * a.units + tid];
  }
  const float last_mass = mass[last];
  const int last_born = born ? born[last] : 0;
  // protection, weight and, in reverse, slot: the smallest goes
  auto rank_of = [](bool safe, unsigned key, int s) {
    return (unsigned long long)safe << 63 | (unsigned long long)key << 31 | (unsigned)(0x7fffffff - s);
  };
  unsigned long long best = ~0ull;
  for (int t0 = tid; t0 < a.N; t0 += THREADS * U) {
    float m[U];
    int age[U];
#pragma unroll
    for (int i = 0; i < U; ++i) m[i] = mass[min(t0 + i * THREADS, last)];
    if (a.protect_from) {
#pragma unroll
      for (int i = 0; i < U; ++i) age[i] = born[min(t0 + i * THREADS, last)];
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int t = t0 + i * THREADS;
      const unsigned long long rank = rank_of(a.protect_from && age[i] >= guard, weight_key(m[i]), t);
      if (t <= last && rank < best) best = rank;
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const unsigned long long other = __shfl_xor(best, o, 64);
    best = other < best ? other : best;
  }
  if (lane == 0) w_best[w] = best;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) best = w_best[i] < best ? w_best[i] : best;
  const int slot = 0x7fffffff - (int)(best & 0x7fffffff);
  if (n <= a.keep || slot == last) return;         // nothing too many, or the last slot itself goes
  if (copies) {
    K[(long)slot * a.units + tid] = kv;
    V[(long)slot * a.units + tid] = vv;
  }
  if (tid == 0) {
    mass[slot] = last_mass;
    if (born) born[slot] = last_born;
  }
  if (a.slab) {
    const int h = a.by_H.mod(bh);
    T *slab = static_cast<T *>(a.slab) + (long)bh * a.nTiles * a.r * TILE;
    const T *row = static_cast<const T *>(a.K) + ((long)bh * a.N_cap + last) * a.d;
    for (int c = tid; c < a.r; c += THREADS)
      slab[((long)(slot / TILE) * a.r + c) * TILE + slot % TILE] = row[min(max(a.idx[h * a.r + c], 0), a.d - 1)];
  }
}

// Bound by memory: 512 pools, about 725 rows of 256 bytes of K and of V each, 80 us = 4.9 TB/s.
constexpr int MOVE_ROWS = 64;      // rows a workgroup of evict_move takes

template <typename T> __global__ __launch_bounds__(256) void evict_move(EvictArgs a) {
  const int bh = a.by_chunks.div(blockIdx.x), j0 = a.by_chunks.mod(blockIdx.x) * MOVE_ROWS;
  const int n = a.count[bh];
  if (j0 >= n) return;
  const int32_t *from = a.moves + (long)bh * 2 * a.most;
  move_rows<T, 256>(a, bh, from, from + a.most, j0, min(n, j0 + MOVE_ROWS));
}

// ---- append of rows -----------------------------------------------------------------------------------
// A workgroup takes 64 rows of one pool, in 16-byte units, four of K and of V in flight a thread.  Bound by memory: 512
// pools, 2048 rows each, 207 us = 5.2 TB/s; a path of five rows to each of 256 pools 3.2 us.
struct AppendArgs {
  const u32x4 *k_rows, *v_rows;
  const int32_t *path, *n_append, *kv_len, *pos, *idx;
  void *slab;
  u32x4 *K, *V;
  float *mass;
  int32_t *born;
  int H, N, N_cap, n_rows, units, d, r, nTiles;
  FastDiv by_H, by_units, by_chunks;
};
constexpr int APPEND_ROWS = 64;    // rows a workgroup takes

template <typename T> __global__ __launch_bounds__(256) void append_rows(AppendArgs a) {
  constexpr int TILE = IG_WAVE * SlabElem<T>::TPL, BATCH = 4;
  const int bh = a.by_chunks.div(blockIdx.x), j0 = a.by_chunks.mod(blockIdx.x) * APPEND_ROWS;
  const int b = a.by_H.div(bh), h = bh - b * a.H;
  const int start = a.kv_len ? min(max(a.kv_len[b], 0), a.N_cap) : a.N;
  const int n = min(a.n_append ? min(max(a.n_append[b], 0), a.n_rows) : a.n_rows, a.N_cap - start);
  const int rows = min(APPEND_ROWS, n - j0);
  if (rows <= 0) return;
  const int32_t *path = a.path ? a.path + (long)b * a.n_rows + j0 : nullptr;
  auto row_of = [&](int j) { return path ? min(max(path[j], 0), a.n_rows - 1) : j0 + j; };
  const long first = (long)bh * a.N_cap + start + j0;        // the first slot written, among all pools' slots
  const int total = rows * a.units;
  for (int u0 = threadIdx.x; u0 < total; u0 += 256 * BATCH) {
    u32x4 kv[BATCH], vv[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int u = min(u0 + 256 * i, total - 1), j = a.by_units.div(u), c = u - j * a.units;
      const long s = (((long)b * a.n_rows + row_of(j)) * a.H + h) * a.units + c;
      kv[i] = a.k_rows[s];
      vv[i] = a.v_rows[s];
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int u = u0 + 256 * i;
      if (u < total) {
        a.K[first * a.units + u] = kv[i];
        a.V[first * a.units + u] = vv[i];
      }
    }
  }
  for (int j = threadIdx.x; j < rows; j += 256) {
    if (a.mass) a.mass[first + j] = 0.f;
    if (a.born) a.born[first + j] = a.pos ? a.pos[b] + j0 + j : start + j0 + j;
  }
  if (a.slab) {
    const T *src = reinterpret_cast<const T *>(a.k_rows);
    T *slab = static_cast<T *>(a.slab) + (long)bh * a.nTiles * a.r * TILE;
    for (int u = threadIdx.x; u < APPEND_ROWS * a.r; u += 256) {
      const int j = u % APPEND_ROWS, c = u / APPEND_ROWS, s = start + j0 + j;
      if (j < rows)
        slab[((long)(s / TILE) * a.r + c) * TILE + s % TILE] =
            src[(((long)b * a.n_rows + row_of(j)) * a.H + h) * a.d + min(max(a.idx[h * a.r + c], 0), a.d - 1)];
    }
  }
}

int most_moves(const ig_desc *d, int keep) { return keep < d->N - keep ? keep : d->N - keep; }
int move_chunks(const ig_desc *d, int keep) { return (most_moves(d, keep) + MOVE_ROWS - 1) / MOVE_ROWS; }
int append_chunks(int n_rows) { return (n_rows + APPEND_ROWS - 1) / APPEND_ROWS; }
// one slot too many at most, in every pool
bool evicts_one(const ig_desc *d, int keep) { return d->N == keep + 1 && d->d * ig_elem_bytes(d->dtype) / 16 <= 256; }

}  // namespace

long ig_evict_threads(const ig_desc *d, int keep) {
  if (d->N <= keep) return 0;
  const long a_pool = d->N > 4096 ? 1024 : (evicts_one(d, keep) ? 256 : 512), moves = evicts_one(d, keep) ? 0 : move_chunks(d, keep) * 256l;
  return d->B * (long)d->H * (a_pool > moves ? a_pool : moves);
}
long ig_append_threads(const ig_desc *d, int n_rows) { return d->B * (long)d->H * append_chunks(n_rows) * 256; }

size_t ig_evict_workspace(const ig_desc *d, int keep) {
  return (size_t)d->B * d->H * (1 + 2 * (size_t)most_moves(d, keep)) * sizeof(int32_t);
}

int ig_launch_evict(ig_ctx *ctx, const ig_desc *d, int keep, const int32_t *kv_len, float *mass, int32_t *born,
                    const int32_t *protect_from, const int32_t *idx, void *slab, void *Kpool, void *Vpool, char *ws,
                    hipStream_t s) {
  const int BH = d->B * d->H, tile = ig_tile_tokens(d->dtype);
  EvictArgs a = {};
  a.kv_len = kv_len, a.protect_from = protect_from, a.idx = idx, a.mass = mass, a.born = born;
  a.K = Kpool, a.V = Vpool, a.slab = slab;
  a.count = reinterpret_cast<int32_t *>(ws), a.moves = a.count + BH;
  a.H = d->H, a.N = d->N, a.N_cap = d->N_cap, a.keep = keep, a.most = most_moves(d, keep);
  a.units = d->d * ig_elem_bytes(d->dtype) / 16, a.d = d->d, a.r = d->r, a.nTiles = (d->N_cap + tile - 1) / tile;
  a.by_H = ig_fast_div(d->H), a.by_units = ig_fast_div(a.units);
  a.by_chunks = ig_fast_div(move_chunks(d, keep));
  const bool one = a.most <= 16;         // few rows a pool: moved by the workgroup that found them
  if (evicts_one(d, keep)) {
    // (256 threads take 8 slots each of 2048; the long pools' 1024 as many of 8192)
#define ONE(T)                                                                                       \
  {                                                                                                  \
    if (d->N <= 4096) {                                                                              \
      auto k = evict_one<T, 256>;                                                                    \
      IG_LAUNCH(ctx, IG_K_EVICT, k, dim3(BH), dim3(256), s, a);                                      \
    } else {                                                                                         \
      auto k = evict_one<T, 1024>;                                                                   \
      IG_LAUNCH(ctx, IG_K_EVICT, k, dim3(BH), dim3(1024), s, a);                                     \
    }                                                                                                \
  }
    if (d->dtype == IG_F16) ONE(half_t) else ONE(float)
    return IG_OK;
  }
#define SELECT(T, THREADS, KPT)                                                                       \
  {                                                                                                  \
    if (one) {                                                                                       \
      auto k = evict_select<T, THREADS, KPT, true>;                                                  \
      IG_LAUNCH(ctx, IG_K_EVICT, k, dim3(BH), dim3(THREADS), s, a);                                  \
    } else {                                                                                         \
      auto k = evict_select<T, THREADS, KPT, false>;                                                 \
      IG_LAUNCH(ctx, IG_K_EVICT, k, dim3(BH), dim3(THREADS), s, a);                                  \
    }                                                                                                \
  }
#define EVICT(T)                                                                                     \
  {                                                                                                  \
    if (d->N <= 512 * 8) SELECT(T, 512, 8)                                                           \
    else if (d->N <= 1024 * 32) SELECT(T, 1024, 32)                                                  \
    else SELECT(T, 1024, 0)                                                                          \
    if (!one) {                                                                                      \
      auto k = evict_move<T>;                                                                        \
      IG_LAUNCH(ctx, IG_K_EVICT, k, dim3((unsigned)(BH * (long)a.by_chunks.d)), dim3(256), s, a);    \
    }                                                                                                \
  }
  if (d->dtype == IG_F16) EVICT(half_t) else EVICT(float)
  return IG_OK;
}

int ig_launch_append_rows(ig_ctx *ctx, const ig_desc *d, int n_rows, const void *k_rows, const void *v_rows,
                          const int32_t *path, const int32_t *n_append, const int32_t *kv_len, const int32_t *pos,
                          const int32_t *idx, void *slab, void *Kpool, void *Vpool, float *mass, int32_t *born,
                          hipStream_t s) {
  const int BH = d->B * d->H, tile = ig_tile_tokens(d->dtype);
  AppendArgs a = {};
  a.k_rows = static_cast<const u32x4 *>(k_rows), a.v_rows = static_cast<const u32x4 *>(v_rows);
  a.path = path, a.n_append = n_append, a.kv_len = kv_len, a.pos = pos, a.idx = idx, a.slab = slab;
  a.K = static_cast<u32x4 *>(Kpool), a.V = static_cast<u32x4 *>(Vpool), a.mass = mass, a.born = born;
  a.H = d->H, a.N = d->N, a.N_cap = d->N_cap, a.n_rows = n_rows, a.d = d->d, a.r = d->r;
  a.units = d->d * ig_elem_bytes(d->dtype) / 16, a.nTiles = (d->N_cap + tile - 1) / tile;
  a.by_H = ig_fast_div(d->H), a.by_units = ig_fast_div(a.units);
  a.by_chunks = ig_fast_div(append_chunks(n_rows));
  const dim3 grid((unsigned)(BH * (long)a.by_chunks.d)), block(256);
  if (d->dtype == IG_F16) {
    auto k = append_rows<half_t>;
    IG_LAUNCH(ctx, IG_K_BUILD, k, grid, block, s, a);
  } else {
    auto k = append_rows<float>;
    IG_LAUNCH(ctx, IG_K_BUILD, k, grid, block, s, a);
  }
  return IG_OK;
}
