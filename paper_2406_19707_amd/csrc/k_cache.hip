// Attention over a whole key / value pool: a prompt, a chunk of one or a single token with the accumulated
// attention weight of every slot, and a tree of drafted tokens over the pool (Section 2.1, softmax(q K^T) V;
// Section 5.3 compares with a cache of a fixed budget, which ranks its entries by the weight that they have received).
#include <type_traits>

#include "cache_device.h"

namespace {

// ---- few query rows, many cached rows ----------------------------------------------------------------
// The R = n_q * group query rows that share a pool (b,h) are taken 16 NT (16 or 32) at a time; the cached rows of a slice
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
// Logits, weights' sums and outputs are float32; in half precision the weights are rounded for the second product, which
// takes no other type at its rate: by at most 2^-11 of themselves, as the output is in the end, where they are above 2^-28 of
// the row's largest (LIFT), and by at most 2^-39 of it below.
// Bound by memory: one token of 16 x 32 heads over 4096 slots 176 us = 6.1 TB/s, of 4 x 40 over 32768 437 us = 6.2 TB/s,
// float32 8 x 32 over 4096 180 us = 6.0 (a copy of 4 GiB: 4.8 TB/s, a read of as much 6.2 at best); 16 nodes over 4096, 128
// pools, 53 us = 5.1.  Small calls are the trips through memory in turn: 32 pools of 777, 5.3 us.
template <typename T, int D, int NT, bool TREE, bool LOGITS>
__global__ __launch_bounds__(256) void attend_stream(StreamArgs a) {
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int TT = HALF ? 32 : 16, MT = TT / 16, CJ = D / 16, RB = 16 * NT;
  constexpr int KCH = D * (int)sizeof(T) / 64;            // 16-byte pieces of a row that a lane holds
  constexpr float LIFT = HALF ? 14.f : 0.f;               // (weights up to 2^14, half precision reaches 2^15)
  constexpr int VT = HALF ? 8 : 4;                        // tokens of a tile that a lane group supplies
  constexpr int VW = CJ * (int)sizeof(T) / 4;             // words of a V row that a lane holds
  // A wave's part of LDS: its outputs at the end (rows of D floats and 16 bytes that set their banks apart), until then
  // logits of up to 16 rows, which wait here because a store before every tile's loads is one more thing that the wait
  // for those waits for (one row, 160 pools of 32768: 501 us in all with stores after every tile, 482 so, 436 without).
  // (At d = 32, in float32 also 64, it is the box that limits the waves of a SIMD, to three.  That costs nothing: with half as
  // large a box 512 pools of 8192, d = 32, 64 and 128, take 116, 211 and 391 us, with this one 116, 208 and 384; float32, 512 of
  // 4096, 108, 200 and 378 with both.)
  constexpr int LDB = D + 4, LOGIT_BOX = LOGITS && NT == 1 ? 3200 : 0, BOX = RB * LDB > LOGIT_BOX ? RB * LDB : LOGIT_BOX;
  __shared__ __attribute__((aligned(16))) float boxes[4][BOX];
  __shared__ float box_m[4][RB], box_l[4][RB];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;

  int work = xcd_order(blockIdx.x, a.per_xcd);
  if (work >= a.total) return;
  // (a head's slices one after the other, the row blocks that share a slice together; a prompt's last rows see most: first)
  const int h = a.by_pair.div(work);
  work -= h * (int)a.by_pair.d;
  const int number = a.by_units.div(work), rb = a.nrb - 1 - a.by_units.mod(work);
  const Span span = span_of<false>(a, number);
  if (span.b < 0) return;
  const int b = span.b, slice = span.slice, bh = b * a.H + h, kv = span.kv, nq = span.nq;

  // What the rows see: slots below their limit, which does not fall from row to row (and, in a tree, the nodes of their
  // masks).
  const int first_row = rb * RB, last_row = min(min(a.R, nq * (int)a.by_group.d), first_row + RB) - 1;
  const bool rows_here = last_row >= first_row;
  const int lim_min = rows_here ? row_limit<TREE>(a, first_row, kv, nq) : 0x7fffffff;
  const int cached = rows_here ? row_limit<TREE>(a, last_row, kv, nq) : 0, cache_tiles = (cached + TT - 1) / TT;
  const int tiles = cache_tiles + (TREE && rows_here ? (nq + TT - 1) / TT : 0);
  const int per = (tiles + span.slices - 1) / span.slices;
  const int t_begin = min(tiles, slice * per);
  int t_end = min(tiles, t_begin + per);
  // (what a slice with the nodes needs to know of them only holds it up where it begins with them)
  unsigned long long seen = 0, masks = 0;
  const bool nodes_here = TREE && t_end > cache_tiles, nodes_first = nodes_here && t_begin + 4 > cache_tiles;
  if (nodes_here) masks = masks_of(a, b, nq);
  auto find_nodes = [&]() __attribute__((always_inline)) {
    seen = nodes_seen(masks, nq);
    if (!seen) t_end = cache_tiles;
  };
  if (nodes_first) find_nodes();

  const T *Kc = static_cast<const T *>(a.K) + (long)bh * a.N_cap * D, *Vc = static_cast<const T *>(a.V) + (long)bh * a.N_cap * D;
  uint4 k[MT][KCH];
  unsigned v[VT][VW];
  // (tokens past the last one that a row sees are read from that one: what they hold is never used, and is finite if that is)
  auto load_k = [&](int tile) __attribute__((always_inline)) {
    const bool drafted = TREE && tile >= cache_tiles;
    const T *base = drafted ? static_cast<const T *>(a.k_tree) + ((long)b * a.n_q * a.by_H.d + h) * D : Kc;
    const long stride = drafted ? (long)a.by_H.d * D : D;
    const int t0 = (drafted ? tile - cache_tiles : tile) * TT, last = (drafted ? nq : cached) - 1;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      int t = min(t0 + (HALF ? 8 * (i >> 2) + 4 * m + (i & 3) : i), last);
      if (TREE && drafted) t = node_read(seen, t);
      const uint4 *src = reinterpret_cast<const uint4 *>(base + t * stride);
#pragma unroll
      for (int c = 0; c < KCH; ++c) k[m][c] = src[c * 4 + g];
    }
  };
  auto load_v = [&](int tile) __attribute__((always_inline)) {
    const bool drafted = TREE && tile >= cache_tiles;
    const T *base = drafted ? static_cast<const T *>(a.v_tree) + ((long)b * a.n_q * a.by_H.d + h) * D : Vc;
    const long stride = drafted ? (long)a.by_H.d * D : D;
    const int t0 = (drafted ? tile - cache_tiles : tile) * TT, last = (drafted ? nq : cached) - 1;
#pragma unroll
    for (int u = 0; u < VT; ++u) {
      int t = min(t0 + VT * g + u, last);
      if (TREE && drafted) t = node_read(seen, t);
      load_words<VW>(base + t * stride + CJ * i, v[u]);
    }
  };

  // A short call is the trips through memory one after the other, so the first tile is asked for with the queries.
  int lim[NT];
  unsigned long long sees[NT];
  bool live[NT];
  uint4 qf[NT][KCH];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = rb * RB + n * 16 + i, iq = a.by_group.div(row), gq = row - iq * (int)a.by_group.d;
    live[n] = row <= last_row;
    lim[n] = live[n] ? row_limit<TREE>(a, row, kv, nq) : 0x7fffffff;
    if (TREE) sees[n] = a.visible[(long)b * a.n_q + min(iq, a.n_q - 1)];
    const uint4 *src = reinterpret_cast<const uint4 *>(
        static_cast<const T *>(a.q) + (((long)b * a.n_q + min(iq, a.n_q - 1)) * a.Hq + h * (int)a.by_group.d + gq) * D);
#pragma unroll
    for (int c = 0; c < KCH; ++c) qf[n][c] = src[c * 4 + g];
  }
  int tile = t_begin + w;
  if (tile < t_end) {
    load_k(tile);
    load_v(tile);
  }
  if (nodes_here && !nodes_first) find_nodes();
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (TREE) sees[n] = live[n] ? sees[n] & low_bits(nq) : 0;
#pragma unroll
    for (int c = 0; c < KCH; ++c) qf[n][c] = flip_sign<T>(qf[n][c], a.flip);
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

  int kept = 0;                                           // tiles in the wave's box of logits
  // (`more` is known at compile time: the waits for a tile's values then leave the next one's keys in flight)
  auto turn = [&](auto more_tiles) __attribute__((always_inline)) {
    constexpr bool more = decltype(more_tiles)::value;
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
    if constexpr (more) load_k(tile + 4);

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
    if constexpr (LOGITS && NT == 1) {
      if (live[0]) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
          *reinterpret_cast<floatx4 *>(boxes[w] + (kept * a.R + i) * TT + VT * g + 4 * m) = s[0][m];
      }
      ++kept;
      if (!more || (kept + 1) * a.R * TT > LOGIT_BOX) {
        // (in the order the rows were written: R rows of a tile, then the wave's next tile)
        lanes_exchange();
        for (int u = lane; u < kept * a.R * (TT / 4); u += 64) {
          const int kr = u / (TT / 4), x = a.by_group.div(kr);       // (one query a sequence: R = group)
          *reinterpret_cast<floatx4 *>(a.logits + ((long)bh * a.R + kr - x * a.R) * a.logits_ld +
                                       (long)(tile - 4 * (kept - 1 - x)) * TT + u % (TT / 4) * 4) =
              *reinterpret_cast<const floatx4 *>(boxes[w] + u * 4);
        }
        lanes_exchange();                                 // (the box is written again, by the next tile or by the outputs)
        kept = 0;
      }
    } else if constexpr (LOGITS) {
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
      top = column_max(top);
      const float ref = fmaxf(m_run[n], lifted(top * a.c, LIFT));
      if (__any(ref > m_run[n])) {
        const float shrink = exp2_fast(m_run[n] - ref);
        l_run[n] *= shrink;
#pragma unroll
        for (int j = 0; j < CJ; ++j) acc[n][j] *= shrink;
        m_run[n] = ref;
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
    if constexpr (more) load_v(tile + 4);
  };
  for (; tile + 4 < t_end; tile += 4) turn(std::true_type());
  if (tile < t_end) turn(std::false_type());

  // ---- the four waves' states joined, and rows out: finished ones to `out`, the states of a slice to the workspace ----
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
      const float by = exp2_fast(box_m[x][at] - m);
      l = fmaf(box_l[x][at], by, l);
      o += *reinterpret_cast<const floatx4 *>(boxes[x] + at * LDB + e) * by;
    }
    if (a.slices == 1) {
      const float inv = inverse_of(l);
      T v[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] = (T)(o[x] * inv);
      store_words<(int)sizeof(T)>(static_cast<T *>(a.out) + (((long)b * a.n_q + iq) * a.Hq + h * (int)a.by_group.d + gq) * D + e, v);
      if (e == 0 && a.stats) a.stats[(long)bh * a.R + row] = make_float2(m, inv);
    } else {
      const long to = ((long)h * a.B * a.slices + number) * a.R + row;
      *reinterpret_cast<floatx4 *>(a.part + to * D + e) = o;
      if (e == 0) a.part_ml[to] = make_float2(m, l);
    }
  }
}

// ---- many query rows, half precision -------------------------------------------------------------------
// The same products on 32x32 matrix instructions: a wave takes 32 query rows, a workgroup 128 (256) that share the
// cached rows' tiles of 64, which come to LDS asynchronously, one (two) ahead.  As above S^T = K Q^T and O^T = V^T P^T,
// so that a query row is one lane of each half wave.  The accumulator of a 32-token block holds, in half h, the
// tokens 8 x + 4 h + 0 .. 3; P^T takes them in that order, and V^T is read through LDS's transposing loads in the
// same one, so the weights never leave their lane.
// The reference of a row's weights only moves when its largest logit has risen by RISE: the row's output, 16 registers for
// every 32 channels, is then scaled only now and then.  It lies LIFT below that logit, so that weights reach 2^15 at most, and
// those above 2^-23 of the largest keep all of half precision's bits (below: to 2^-34 of it).
// Bound by the vector and matrix units together: 8 x 32 heads of 2048 tokens, d = 128, 355 us = 775 TFLOP/s of what is
// seen (a library product of 8192 squared reaches 1107), the matrix units busy for 0.41 of the cycles and the vector units
// for 0.52; d = 64 207 us, d = 256 and half the heads 433 us.  One half block after the other, row blocks not in pairs: 443 us.
constexpr float RISE = 6.f, PROMPT_LIFT = 9.f;
constexpr int PROMPT_KEYS = 64;

template <int D, int NW, bool TREE> __global__ __launch_bounds__(NW * 64, D <= 128 ? 2 : 1) void attend_prompt(StreamArgs a) {
  constexpr int KS = D / 16, OB = D / 32, PC = D / 8, TK = PROMPT_KEYS, ROWS = NW * 32;
  constexpr int SLOTS = NW == 8 ? 3 : 2, AHEAD = SLOTS - 1;      // tiles in LDS, and how many of them ahead of their use
  constexpr int LOADS = PC / NW;                                  // of a wave, for a tile of K or of V
  static_assert(LOADS >= 1, "every wave loads a part of a tile");
  __shared__ __attribute__((aligned(16))) half_t tiles[SLOTS][2][TK * D];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 31, hb = lane >> 5;
  int work = xcd_order(blockIdx.x, a.per_xcd);
  if (work >= a.total) return;
  const int h = a.by_pair.div(work);
  work -= h * (int)a.by_pair.d;
  const int number = a.by_units.div(work), unit = a.by_units.mod(work);
  const Span span = span_of<false>(a, number);
  if (span.b < 0) return;
  const int b = span.b, slice = span.slice, bh = b * a.H + h, G = (int)a.by_group.d, kv = span.kv, nq = span.nq;

  // what this lane fetches of every tile: this piece of this row first, then of 64 / PC rows further on, ..
  const unsigned from_row = w * (64 / NW) + lane / PC, from_piece = (lane % PC) ^ piece_swap<D>(from_row);
  // (a tree's masks leave no registers for all of these: there they are made from the first ones)
  unsigned k_at[KS], v_at[OB][2];
#pragma unroll
  for (int k = 0; k < KS; ++k) k_at[k] = row_offset<D>(lane, k);
#pragma unroll
  for (int o = 0; o < OB; ++o)
#pragma unroll
    for (int x = 0; x < 2; ++x) v_at[o][x] = column_offset<D>(lane, o, x);

  // one row block; in a paired call the last with the first, the last but one with the second, ..
  for (int turn = 0; turn < (a.paired ? 2 : 1); ++turn) {
    const int rb = turn ? unit : a.nrb - 1 - unit;        // (a prompt's last rows see most: first)
    if (turn) {
      if (2 * unit >= a.nrb - 1) break;
      __syncthreads();                                    // the other waves are done with the tiles
    }
    const int row = rb * ROWS + w * 32 + i, iq = a.by_group.div(row), gq = row - iq * G;
    const bool live = row < a.R && iq < nq;
    const int lim = live ? row_limit<TREE>(a, row, kv, nq) : 0x7fffffff;
    const unsigned long long sees = TREE && live ? a.visible[(long)b * a.n_q + iq] & low_bits(nq) : 0;
    const long row_at = (((long)b * a.n_q + min(iq, a.n_q - 1)) * a.Hq + h * G + gq) * D;
    // (limits do not fall from row to row)
    const int first_row = rb * ROWS + w * 32, lim_min = row_limit<TREE>(a, first_row, kv, nq);
    // (what the row block's last live row sees)
    const int last_row = min(min(a.R, nq * G), (rb + 1) * ROWS) - 1;
    const int most = last_row < rb * ROWS ? 0 : row_limit<TREE>(a, last_row, kv, nq);
    const int cache_tiles = (most + TK - 1) / TK;
    const int tiles_all = cache_tiles + (TREE && last_row >= rb * ROWS ? (nq + TK - 1) / TK : 0);
    const int per = (tiles_all + span.slices - 1) / span.slices;
    const int t_begin = min(tiles_all, slice * per);
    int t_end = min(tiles_all, t_begin + per);
    // (what a slice with the nodes needs to know of them only holds it up where it begins with them)
    unsigned long long seen = 0, masks = 0;
    const bool nodes_here = TREE && t_end > cache_tiles, nodes_first = nodes_here && t_begin + AHEAD > cache_tiles;
    if (nodes_here) masks = masks_of(a, b, nq);
    auto find_nodes = [&]() __attribute__((always_inline)) {
      seen = nodes_seen(masks, nq);
      if (!seen) t_end = cache_tiles;
    };
    if (nodes_first) find_nodes();

    half8 qf[KS];
    {
      const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const half_t *>(a.q) + row_at);
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(half8, flip_sign<half_t>(src[2 * s + hb], a.flip));
    }
    // tile `tile` of K or V into a slot (past the last one: the last one again, so that every turn has as many loads)
    auto fetch = [&](const void *pool, const void *nodes, int tile, half_t *to) __attribute__((always_inline)) {
      tile = min(tile, t_end - 1);
      const unsigned r0 = opaque(from_row);
      if (TREE && tile >= cache_tiles) {                  // (64 nodes at most: one tile)
        const char *base = static_cast<const char *>(nodes) + ((long)b * a.n_q * a.by_H.d + h) * D * 2;
#pragma unroll
        for (int x = 0; x < LOADS; ++x)
          load_to_lds(base, (unsigned)(node_read(seen, min((int)r0 + x * (64 / PC), nq - 1)) * (int)a.by_H.d * D * 2) +
                                (from_piece ^ piece_swap<D>(x * (64 / PC))) * 16, to + (w * LOADS + x) * 512);
        return;
      }
      const char *base = static_cast<const char *>(pool) + ((long)bh * a.N_cap + (long)tile * TK) * D * 2;
      const int last = most - 1 - tile * TK;
#pragma unroll
      for (int x = 0; x < LOADS; ++x)
        load_to_lds(base, (unsigned)(min((int)r0 + x * (64 / PC), last) * D * 2) + (from_piece ^ piece_swap<D>(x * (64 / PC))) * 16,
                    to + (w * LOADS + x) * 512);
    };

    floatx16 acc[OB];
#pragma unroll
    for (int o = 0; o < OB; ++o)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[o][e] = 0.f;
    float ref = NOTHING_SEEN, sums[4] = {0.f, 0.f, 0.f, 0.f};       // (four sums: no chain of dependent additions)
    floatx16 sA = {}, sB = {};
    half8 pA[2], pB[2];

    // The 32-token half blocks of the tiles are a pipeline: while the weights of one are worked out on the vector
    // units, the matrix units take the logits of the next and the output of the one before.
    //   now: logits in, weights out (half `now_half` of tile `now_tile`); next: the logits of rows `next_row` ..
    //   of tile K; out: acc += the weights `old` times rows `old_row` .. of tile V
    auto half_step = [&](auto has_now, auto has_next, auto has_old, const floatx16 &now, int now_tile, int now_half,
                         half8 (&weights)[2], floatx16 &next, const half_t *K, int next_row, const half8 (&old)[2],
                         const half_t *V, int old_row) __attribute__((always_inline)) {
      constexpr bool NOW = decltype(has_now)::value, NEXT = decltype(has_next)::value, OLD = decltype(has_old)::value;
      half8 kf[KS];
      uint2 vt[2][OB][2];
      if constexpr (NEXT) {
        const unsigned first = TREE ? opaque(k_at[0]) : 0;
#pragma unroll
        for (int k = 0; k < KS; ++k) kf[k] = row_piece(K + next_row * D, TREE ? first ^ k << 5 : k_at[k]);
      }
      if constexpr (OLD) {
        const unsigned first = TREE ? opaque(v_at[0][0]) : 0;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int o = 0; o < OB; ++o)
#pragma unroll
            for (int x = 0; x < 2; ++x)
              vt[k][o][x] = column_rows<D>(V + (old_row + k * 16) * D, TREE ? first ^ (o << 6 | x << 5) : v_at[o][x], x);
      }
      floatx16 s;
      float shrink = 1.f;
      bool rises = false;
      if constexpr (NOW) {
        s = now;
        const bool drafted = TREE && now_tile >= cache_tiles;
        const int t0 = (drafted ? now_tile - cache_tiles : now_tile) * TK + now_half * 32;
        if (drafted) {
          const unsigned bits = (unsigned)(sees >> (now_half * 32)) >> opaque(hb * 4);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!(bits >> ((e / 4) * 8 + e % 4) & 1)) s[e] = -INFINITY;
        } else if (t0 + 32 > lim_min) {
          const int mine = t0 + (int)opaque(hb * 4);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (mine + ((e / 4) * 8 + e % 4) >= lim) s[e] = -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = __builtin_elementwise_maximum(top, s[e]);
        top = lifted(both_max(top) * a.c, PROMPT_LIFT);
        const float to = top > ref + RISE ? top : ref;
        rises = __any(to != ref);
        shrink = exp2_fast(ref - to);
        ref = to;
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[e] *= shrink;
      }
      if constexpr (NEXT) {
#pragma unroll
        for (int e = 0; e < 16; ++e) next[e] = 0.f;
      }
      // (one product of each kind after the other, with the vector work between them)
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        if constexpr (NEXT) {
#pragma unroll
          for (int k = x * KS / 8; k < (x + 1) * KS / 8; ++k)
            next = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[k], qf[k], next, 0, 0, 0);
        }
        if constexpr (OLD) {
#pragma unroll
          for (int y = x * 2 * OB / 8; y < (x + 1) * 2 * OB / 8; ++y) {
            const int k = y / OB, o = y % OB;
            const uint4 v = make_uint4(vt[k][o][0].x, vt[k][o][0].y, vt[k][o][1].x, vt[k][o][1].y);
            acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, v), old[k], acc[o], 0, 0, 0);
          }
        }
        if constexpr (NOW) {
#pragma unroll
          for (int e = 2 * x; e < 2 * x + 2; ++e) {
            const float p = exp2_fast(fmaf(s[e], a.c, -ref));
            sums[e % 4] += p;
            weights[e / 8][e % 8] = (half_t)p;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) keep_here(sums[e]);      // (not put off: the weights' registers are needed)
      if (NOW && rises) {
#pragma unroll
        for (int o = 0; o < OB; ++o) acc[o] *= shrink;
      }
    };
    typedef std::true_type Y;
    typedef std::false_type N;
    if (t_end > t_begin) {
      fetch(a.K, a.k_tree, t_begin, tiles[0][0]);
      if constexpr (AHEAD == 2) {
        fetch(a.K, a.k_tree, t_begin + 1, tiles[1][0]);
        fetch(a.V, a.v_tree, t_begin, tiles[0][1]);
      }
      if (nodes_here && !nodes_first) find_nodes();
      const int turns = t_end - t_begin;
      // Turn r: the logits of tile r, the weights of its first half and of the last tile's second half, the last tile's
      // output.  Slots go round: tile r of K or V is in slot r % SLOTS.
      auto begin_turn = [&](int r, auto slot) __attribute__((always_inline)) {
        constexpr int S = decltype(slot)::value;
        wait_for_lds_loads<(AHEAD - 1) * 2 * LOADS>();    // this turn's tiles are there ...
        __syncthreads();                                  // ... in every wave's part, and the last turn's slots are free
        fetch(a.K, a.k_tree, t_begin + r + AHEAD, tiles[(S + AHEAD) % SLOTS][0]);
        fetch(a.V, a.v_tree, t_begin + r + AHEAD - 1, tiles[(S + AHEAD - 1) % SLOTS][1]);
      };
      auto turn_of = [&](int r, auto slot) __attribute__((always_inline)) {
        constexpr int S = decltype(slot)::value;
        begin_turn(r, slot);
        const half_t *K = tiles[S][0], *V = tiles[(S + SLOTS - 1) % SLOTS][1];
        half_step(Y(), Y(), Y(), sB, t_begin + r - 1, 1, pB, sA, K, 0, pA, V, 0);
        half_step(Y(), Y(), Y(), sA, t_begin + r, 0, pA, sB, K, 32, pB, V, 32);
      };
      begin_turn(0, std::integral_constant<int, 0>());
      half_step(N(), Y(), N(), sB, 0, 0, pB, sA, tiles[0][0], 0, pA, tiles[0][1], 0);
      half_step(Y(), Y(), N(), sA, t_begin, 0, pA, sB, tiles[0][0], 32, pB, tiles[0][1], 0);
      typedef std::integral_constant<int, 1> S1;
      typedef std::integral_constant<int, 2 % SLOTS> S2;
      typedef std::integral_constant<int, 0> S0;
      int r = 1;
      for (; r + SLOTS - 1 < turns; r += SLOTS) {
        turn_of(r, S1());
        turn_of(r + 1, S2());
        if constexpr (SLOTS == 3) turn_of(r + 2, S0());
      }
      if (r < turns) turn_of(r, S1());
      if (SLOTS == 3 && r + 1 < turns) turn_of(r + 1, S2());
      wait_for_lds_loads<0>();
      __syncthreads();
      const half_t *V = tiles[(turns - 1) % SLOTS][1];
      half_step(Y(), N(), Y(), sB, t_end - 1, 1, pB, sA, V, 0, pA, V, 0);
      half_step(N(), N(), Y(), sA, 0, 0, pA, sB, V, 0, pB, V, 32);
    }

    if (!live) continue;
    const float sum = both_sum((sums[0] + sums[1]) + (sums[2] + sums[3]));
    const float inv = inverse_of(sum);
    if (a.slices == 1) {
      half_t *to = static_cast<half_t *>(a.out) + row_at;
#pragma unroll
      for (int o = 0; o < OB; ++o)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          half_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (half_t)(acc[o][x * 4 + e] * inv);
          store_words<2>(to + o * 32 + x * 8 + hb * 4, v);
        }
      if (hb == 0 && a.stats) a.stats[(long)bh * a.R + row] = make_float2(ref, inv);
    } else {
      const long at = ((long)h * a.B * a.slices + number) * a.R + row;
#pragma unroll
      for (int o = 0; o < OB; ++o)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          *reinterpret_cast<floatx4 *>(a.part + at * D + o * 32 + x * 8 + hb * 4) =
              floatx4{acc[o][x * 4], acc[o][x * 4 + 1], acc[o][x * 4 + 2], acc[o][x * 4 + 3]};
      if (hb == 0) a.part_ml[at] = make_float2(ref, sum);
    }
  }
}

// ---- joining the slices, and the weights of single-token calls ------------------------------------------
// A workgroup takes 256 E / d rows of a pool, E elements a thread, and, where logits were kept, 1024 slots of it:
// mass[t] += sum over the rows of exp2(c s - ref) / sum.  Small calls are a chain of trips through memory, so slices are
// taken eight at a time, all their loads together, and a slot's weight and first logit are asked for before the sums are
// known (32 pools of 777 slots, 7 slices: 8.6 -> 4.3 us; 160 pools of 32768: 19 us for 63 MB).
template <int E> struct Joined {
  float ref, sum, out[E ? E : 1];
};
// the row's state over all slices, and elements e .. e + E - 1 of its output before the division
template <int E> __device__ __forceinline__ Joined<E> join_row(const StreamArgs &a, int h, const Span &span, int row, int D, int e) {
  constexpr int U = 8;
  Joined<E> j = {NOTHING_SEEN, 0.f, {}};
  for (int s0 = 0; s0 < span.slices; s0 += U) {
    float2 ml[U];
    unsigned o[U][E ? E : 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long at = ((long)h * a.B * a.slices + span.first + min(s0 + u, span.slices - 1)) * a.R + row;
      ml[u] = a.part_ml[at];
      if constexpr (E > 0) load_words<E>(a.part + at * D + e, o[u]);
    }
    float ref = j.ref;
#pragma unroll
    for (int u = 0; u < U; ++u) ref = fmaxf(ref, ml[u].x);          // (the last slice again and again is the same)
    const float shrink = exp2_fast(j.ref - ref);          // (of outputs)
    j.sum = add_scaled(0.f, j.sum, j.ref - ref), j.ref = ref;
#pragma unroll
    for (int k = 0; k < E; ++k) j.out[k] *= shrink;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + u < span.slices) {
        const float by = exp2_fast(ml[u].x - ref);
        j.sum = add_scaled(j.sum, ml[u].y, ml[u].x - ref);
#pragma unroll
        for (int k = 0; k < E; ++k) j.out[k] = fmaf(__uint_as_float(o[u][k]), by, j.out[k]);
      }
  }
  return j;
}

template <typename T, int E, bool LOGITS>
__global__ __launch_bounds__(256) void attend_join(StreamArgs a, float *mass, int D, FastDiv by_chunks, FastDiv by_threads) {
  constexpr int SLOTS = 1024, U = SLOTS / 256;
  __shared__ float2 stat[32];                              // (LOGITS: R <= 32)
  const int bh = by_chunks.div(blockIdx.x), x = by_chunks.mod(blockIdx.x), tid = threadIdx.x;
  const int b = a.by_H.div(bh), h = bh - b * (int)a.by_H.d, G = (int)a.by_group.d;
  const Span span = span_of<true>(a, b);
  const int kv = span.kv, nq = span.nq;
  float *m = mass + (long)bh * a.N_cap;
  const float *logits = a.logits + (long)bh * a.R * a.logits_ld;
  float before[U], first[U];
  const bool slots = LOGITS && x * SLOTS < kv && nq > 0;
  if (slots) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(x * SLOTS + u * 256 + tid, kv - 1);
      before[u] = m[t];
      first[u] = logits[t];
    }
  }
  if (a.slices > 1) {
    const int mine = by_threads.div(tid), row = x * by_threads.div(256) + mine, e = (tid - mine * (int)by_threads.d) * E;
    if (row < nq * G) {
      const Joined<E> j = join_row<E>(a, h, span, row, D, e);
      const float inv = inverse_of(j.sum);
      const int iq = a.by_group.div(row), gq = row - iq * G;
      T *to = static_cast<T *>(a.out) + (((long)b * a.n_q + iq) * a.Hq + h * G + gq) * D + e, v[E];
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] = (T)(j.out[k] * inv);
      if constexpr (E == 1) *to = v[0];
      else store_words<E * (int)sizeof(T) / 4>(to, v);
      if (a.stats && e == 0) a.stats[(long)bh * a.R + row] = make_float2(j.ref, inv);
    }
  }
  if (!slots) return;
  if (tid < a.R) {
    if (a.slices > 1) {
      const Joined<0> j = join_row<0>(a, h, span, tid, D, 0);
      stat[tid] = make_float2(j.ref, inverse_of(j.sum));
    } else {
      stat[tid] = a.stats[(long)bh * a.R + tid];
    }
  }
  __syncthreads();
  float sum[U];
#pragma unroll
  for (int u = 0; u < U; ++u) sum[u] = exp2_fast(fmaf(first[u], a.c, -stat[0].x)) * stat[0].y;
  for (int row = 1; row < a.R; ++row) {
    float s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) s[u] = logits[row * a.logits_ld + min(x * SLOTS + u * 256 + tid, kv - 1)];
    const float2 st = stat[row];
#pragma unroll
    for (int u = 0; u < U; ++u) sum[u] = fmaf(exp2_fast(fmaf(s[u], a.c, -st.x)), st.y, sum[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = x * SLOTS + u * 256 + tid;
    if (t < kv) m[t] = before[u] + sum[u];
  }
}

// ---- the weights of many query rows ------------------------------------------------------------------
// Float32: a workgroup keeps 32 cached keys (d = 256: 16) as the rows of S^T = K Q^T; its waves take turns at the
// query rows that see them, 16 at a time with the next 16 asked for: mass[t] += sum over rows of
// exp2(c s - ref) / sum, with the rows' final references and sums.  2 x 16 heads of
// 1024 tokens, d = 128, 108 us = 40 TFLOP/s, a quarter of what a library product reaches in float32: every 32 keys read the query
// rows again, and two waves a SIMD with 16 rows asked for ahead have to hide that.  4 heads of 512, d = 64, 9.6 us (32 us with a
// wave for every 16 keys and nothing asked for ahead).
template <int D> constexpr int mass_keys() { return D <= 128 ? 32 : 16; }
template <int D> __global__ __launch_bounds__(256) void attend_mass(StreamArgs a, float *mass, FastDiv by_chunks) {
  constexpr int MT = mass_keys<D>() / 16, KCH = D / 16;
  __shared__ float part[4][mass_keys<D>()];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int bh = by_chunks.div(blockIdx.x), x = by_chunks.mod(blockIdx.x);
  const int b = a.by_H.div(bh), h = bh - b * (int)a.by_H.d, G = (int)a.by_group.d;
  const int kv = length_of(a.kv_len, b, a.N, a.N_cap), nq = length_of(a.q_len, b, a.n_q, a.n_q);
  const int t0 = x * mass_keys<D>();
  if (t0 >= kv) return;
  const float *Kc = static_cast<const float *>(a.K) + (long)bh * a.N_cap * D;
  uint4 k[MT][KCH], q[KCH];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const uint4 *src = reinterpret_cast<const uint4 *>(Kc + (long)min(t0 + m * 16 + i, kv - 1) * D);
#pragma unroll
    for (int c = 0; c < KCH; ++c) k[m][c] = flip_sign<float>(src[c * 4 + g], a.flip);
  }
  float sum[MT][4] = {};
  // the first query that sees slot t0 is number t0 - (kv - nq)
  const int rows = nq * G, first = max(0, t0 - (kv - nq)) * G;
  float2 st;
  int iq;
  auto ask = [&](int r0) __attribute__((always_inline)) {
    const int row = min(r0 + i, rows - 1);
    iq = a.by_group.div(row);
    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const float *>(a.q) + (((long)b * a.n_q + iq) * a.Hq + h * G + row - iq * G) * D);
#pragma unroll
    for (int c = 0; c < KCH; ++c) q[c] = src[c * 4 + g];
    st = a.stats[(long)bh * a.R + row];
  };
  int r0 = first + 16 * w;
  if (r0 < rows) ask(r0);
  for (; r0 < rows; r0 += 64) {
    floatx4 s[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) s[m] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KCH; ++c)
#pragma unroll
      for (int m = 0; m < MT; ++m) s[m] = dot_step<float>(k[m][c], q[c], s[m]);
    const float ref = st.x, inv = st.y;
    const int lim = r0 + i < rows ? kv - nq + iq + 1 : 0;
    if (r0 + 64 < rows) ask(r0 + 64);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (t0 + m * 16 + 4 * g + r < lim) sum[m][r] = fmaf(exp2_fast(fmaf(s[m][r], a.c, -ref)), inv, sum[m][r]);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float all = row16_sum(sum[m][r]);
      if (i == 0) part[w][m * 16 + 4 * g + r] = all;
    }
  __syncthreads();
  const int e = threadIdx.x;
  if (e < mass_keys<D>() && t0 + e < kv) mass[(long)bh * a.N_cap + t0 + e] += (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
}

// Half precision: a wave keeps 64 keys, a workgroup 256, and the query rows
// come through LDS 64 at a time, one tile ahead.  As in attend_prompt it is a pipeline: while the weights of 32 rows
// and 32 keys are worked out (an exponential and two fused multiply-adds a pair), the matrix units take the next
// logits.  The logits are worked out again because no weight is known before a row's last slot.  8 x 32 heads of 2048: 195 us,
// vector units busy for 0.63 of the cycles and matrix units for 0.37; in 32-row tiles without the pipeline 274 us, with 16
// query rows a product and no LDS 1149 us.
constexpr int MASS_KEYS = 256, MASS_ROWS = 64;
template <int D> __global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void prompt_mass(StreamArgs a, float *mass) {
  constexpr int KS = D / 16, PC = D / 8;
  __shared__ __attribute__((aligned(16))) half_t tiles[2][MASS_ROWS * D];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 31, hb = lane >> 5;
  const int work = xcd_order(blockIdx.x, a.per_xcd);
  if (work >= a.total) return;
  const int bh = a.by_pair.div(work), unit = work - bh * (int)a.by_pair.d;
  const int b = a.by_H.div(bh), h = bh - b * (int)a.by_H.d, G = (int)a.by_group.d;
  const int kv = length_of(a.kv_len, b, a.N, a.N_cap), nq = length_of(a.q_len, b, a.n_q, a.n_q);
  const int rows = nq * G;
  const unsigned from_row = w * 16 + lane / PC, from_piece = (lane % PC) ^ piece_swap<D>(from_row);
  unsigned q_at[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) q_at[k] = row_offset<D>(lane, k);

  // one block of keys; in a paired call the first with the last, the second with the last but one, ..
  for (int turn = 0; turn < (a.paired ? 2 : 1); ++turn) {
    const int kb = turn ? a.nrb - 1 - unit : unit;        // (a prompt's first keys are seen by most rows: first)
    if (turn) {
      if (2 * unit >= a.nrb - 1) break;
      __syncthreads();                                    // the other waves are done with the tiles
    }
    if (kb * MASS_KEYS >= kv) continue;
    const int t0 = kb * MASS_KEYS + w * 64;
    // the first query that sees slot t is number t - (kv - nq)
    const int first = max(0, kb * MASS_KEYS - (kv - nq)) * G;
    const int tiles_n = (max(0, rows - first) + MASS_ROWS - 1) / MASS_ROWS;
    half8 kf[2][KS];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const half_t *src = static_cast<const half_t *>(a.K) + ((long)bh * a.N_cap + min(t0 + m * 32 + i, kv - 1)) * D;
#pragma unroll
      for (int k = 0; k < KS; ++k) kf[m][k] = __builtin_bit_cast(half8, flip_sign<half_t>(reinterpret_cast<const uint4 *>(src)[2 * k + hb], a.flip));
    }
    auto fetch = [&](int tile, half_t *to) __attribute__((always_inline)) {
      if (tile >= tiles_n) return;
      const int r0 = first + tile * MASS_ROWS, iq0 = a.by_group.div(r0);
      const half_t *q0 = static_cast<const half_t *>(a.q) + (((long)b * a.n_q + iq0) * a.Hq + h * G) * D;
      const int mine = r0 + (int)opaque(from_row);
#pragma unroll
      for (int x = 0; x < PC / 4; ++x) {
        const int row = min(mine + x * (64 / PC), rows - 1), iq = a.by_group.div(row);
        load_to_lds(q0, (unsigned)(((iq - iq0) * a.Hq + row - iq * G) * D) * 2 + (from_piece ^ piece_swap<D>(x * (64 / PC))) * 16,
                    to + (w * (PC / 4) + x) * 512);
      }
    };
    // a half tile's row of this lane: what its weights are relative to, 1 / their sum, and the slots it sees
    struct Row {
      float ref, inv;
      int seen;
    };
    auto row_of = [&](int tile, int half, float2 st) __attribute__((always_inline)) {
      const int r = first + tile * MASS_ROWS + half * 32 + i;
      const bool there = r < rows;                        // (else weights of zero)
      return Row{there ? st.x : INFINITY, there ? st.y : 0.f, kv - nq + a.by_group.div(min(r, rows - 1)) + 1};
    };
    float2 st[2], st_now[2];                              // of the next tile, asked for with it, and of this one
    auto ask = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
        st[half] = a.stats[(long)bh * a.R + min(first + tile * MASS_ROWS + half * 32 + i, rows - 1)];
    };
    floatx16 sums[2] = {}, sA = {}, sB = {};
    half8 qf[KS];
    auto read_rows = [&](const half_t *Q) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[k] = row_piece(Q, q_at[k]);
    };
    // weights of the logits `now` (row, keys m) added to the sums, while `next` becomes the logits of the rows in qf and keys n
    auto step = [&](auto has_now, auto has_next, const floatx16 &now, const Row &row, int m, floatx16 &next, int n) __attribute__((always_inline)) {
      constexpr bool NOW = decltype(has_now)::value, NEXT = decltype(has_next)::value;
      floatx16 s = now;
      if constexpr (NOW) {
        if (__any(row.seen < t0 + m * 32 + 32)) {
          const int mine = t0 + m * 32 + (int)opaque(hb * 4);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (mine + ((e / 4) * 8 + e % 4) >= row.seen) s[e] = -INFINITY;
        }
      }
      if constexpr (NEXT) {
#pragma unroll
        for (int e = 0; e < 16; ++e) next[e] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) next = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[n][k], qf[k], next, 0, 0, 0);
      }
      if constexpr (NOW) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[m][e] = fmaf(exp2_fast(fmaf(s[e], a.c, -row.ref)), row.inv, sums[m][e]);
        keep_here(sums[m]);
      }
    };
    typedef std::true_type Y;
    typedef std::false_type N;
    if (tiles_n > 0) {
      fetch(0, tiles[0]);
      ask(0);
      wait_for_lds_loads<0>();
      __syncthreads();
      Row rA = row_of(0, 0, st[0]), rB = row_of(0, 1, st[1]);
      auto turn_of = [&](auto has_last, int tile, half_t *q, half_t *q_free) __attribute__((always_inline)) {
        fetch(tile + 1, q_free);
        ask(tile + 1);
        read_rows(q);
        step(has_last, Y(), sB, rB, 1, sA, 0);
        if (decltype(has_last)::value) rA = row_of(tile, 0, st_now[0]), rB = row_of(tile, 1, st_now[1]);
        step(Y(), Y(), sA, rA, 0, sB, 1);
        read_rows(q + 32 * D);
        step(Y(), Y(), sB, rA, 1, sA, 0);
        step(Y(), Y(), sA, rB, 0, sB, 1);
      };
      auto next_tile = [&]() __attribute__((always_inline)) {
        wait_for_lds_loads<0>();                             // the tile is there ...
        __syncthreads();                                  // ... in every wave's part, and the other slot is free
        st_now[0] = st[0], st_now[1] = st[1];
      };
      turn_of(N(), 0, tiles[0], tiles[1]);
      int tile = 1;
      for (; tile + 1 < tiles_n; tile += 2) {
        next_tile();
        turn_of(Y(), tile, tiles[1], tiles[0]);
        next_tile();
        turn_of(Y(), tile + 1, tiles[0], tiles[1]);
      }
      if (tile < tiles_n) {
        next_tile();
        turn_of(Y(), tile, tiles[1], tiles[0]);
      }
      step(Y(), N(), sB, rB, 1, sA, 0);
    }
    // the 32 lanes of a half wave added up; lane i then keeps the sum of register i
    float mine = 0.f;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float v = row16_sum(sums[m][e]);
        v += __shfl_xor(v, 16, 64);
        if (i == m * 16 + e) mine = v;
      }
    const int t = t0 + (i / 16) * 32 + ((i % 16) / 4) * 8 + hb * 4 + i % 4;
    if (t < kv) mass[(long)bh * a.N_cap + t] += mine;
  }
}

int div_up(long n, long d) { return (int)((n + d - 1) / d); }

// Query rows a workgroup of attend_stream takes: 16 or 32.  (With 64 the registers run out: float32, 1024 rows over as
// many, 121 us with 32 and 163 us with 64.)  In half precision attend_prompt takes over from there: trees of 33 to 64 nodes
// over 4096, 128 pools, 62 to 67 us there, 101 to 105 us here in two blocks.  Up to 32 nodes: the same pools with 17, 24 and
// 32, 63, 62 and 63 us here, 72, 63 and 61 there; 512 pools 185 to 187 here, 203 to 218 there; d = 64, 128 pools, 29 to 30
// here, 35 there; only small calls the other way round (8 pools of 1024: 12.5 to 13.5 here, 11 to 12 there).
// (d = 256: 16 here, and from 17 rows on in half precision there.)
int row_block(const ig_desc *d, long R) { return R <= 16 || d->d > 128 ? 16 : 32; }
bool many_rows(const ig_desc *d, long R) { return d->dtype == IG_F16 && R > (d->d > 128 ? 16 : 32); }

// The same for attend_prompt.  Eight waves, two tiles ahead, where most of what the rows see is seen by all of them and
// there are rows for more than four (317 x 4 query rows over up to 9001: 225 against 235 us, trees of 63 x 4 nodes over
// 8191: 97 against 106, before slices went by length); four for prompts, where a block of 256 rows works out more that its
// first rows do not see (2048 over 2048: 397 against 367 us).
int prompt_rows(const ig_desc *d, const CacheCall &c) {
  return d->d >= 64 && d->d <= 128 && (long)c.n_q * c.group > 128 && (c.k_tree || 2 * (long)c.n_q <= d->N) ? 256 : 128;
}

// Slices the cached rows of a pool are cut into: the number for which the last workgroups end first, if a turn (64
// rows of attend_prompt, four waves' tiles of attend_stream) takes a unit of time, a workgroup two more to start and
// to leave its state, the join three for every eight slices, and a compute unit holds eight waves.  (8 pools of 32768: 31 us
// with 24 slices, 35 with 16, 36 with 64; 32 of 777: 8.8 with 8, 9.7 with 4, 11.2 with 16, 13.6 with one.  Four sequences
// of up to 9001 with 1268 query rows for each of 8 pools: 3 slices of 320 row blocks 1.5 times as fast as 2, which leave the
// second round a quarter full.)  Eight waves is what d = 128 holds, up to 16 rows or from 33 on, and where all of this was
// measured.  With 17 to 32 rows there, and at d = 256, it holds four, at d = 32 and 64 from 8 to 32: what the model calls a
// round is then off by as much.
// Never more than four rounds of workgroups, so that the states they leave are bounded (ig_cache_reserve_bytes).
constexpr long ROUNDS = 4;
long slots_of(int prompt_rows) { return prompt_rows == 256 ? 256 : 512; }
int slices_of(const ig_desc *d, int prompt_rows, long nrb, int n_keys) {
  const long groups = d->B * (long)d->H * nrb, slots = slots_of(prompt_rows);
  const long turns = div_up(n_keys, prompt_rows ? 64 : (d->dtype == IG_F16 ? 128 : 64));
  long best = 1, best_cost = -1;
  for (long s = 1; s <= MOST_SLICES && s <= turns && (s == 1 || groups * s <= ROUNDS * slots); ++s) {
    const long cost = div_up(groups * s, slots) * (div_up(turns, s) + 2) + (s > 1 ? 3 * div_up(s, 8) : 0);
    if (best_cost < 0 || cost < best_cost) best = s, best_cost = cost;
  }
  return (int)best;
}

}  // namespace

// Whether the logits of a call are kept for the weights (one query a sequence) instead of being worked out
// again from the keys.
static bool keeps_logits(const CacheCall &c, const CachePlan &p) { return c.mass && c.n_q == 1 && p.nrb == 1 && !p.prompt; }

CachePlan ig_cache_plan(const ig_desc *d, const CacheCall &c) {
  CachePlan p;
  const long R = (long)c.n_q * c.group, BH = (long)d->B * d->H;
  p.prompt = many_rows(d, R);
  p.rb = p.prompt ? prompt_rows(d, c) : row_block(d, R);
  p.nrb = div_up(R, p.rb);
  p.slices = slices_of(d, p.prompt ? p.rb : 0, p.nrb, d->N + (c.k_tree ? c.n_q : 0));
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  p.logits_ld = ((long)d->N + 63) / 64 * 64;
  // the rows' launch, the join's (of many workgroups only without slices, for kept logits) and the weights'
  const bool logits = keeps_logits(c, p);
  const int mass_block = d->dtype == IG_F16 ? MASS_KEYS : (d->d <= 128 ? mass_keys<128>() : mass_keys<256>());
  p.threads = (BH * p.slices * p.nrb + 8) * (p.prompt && p.rb == 256 ? 512 : 256);
  const long join = logits ? BH * div_up(d->N, 1024) * 256 : 0, mass = c.mass && !logits ? (BH * div_up(d->N, mass_block) + 8) * 256 : 0;
  p.threads = p.threads > join ? p.threads : join;
  p.threads = p.threads > mass ? p.threads : mass;
  p.stats_at = take(c.mass ? BH * R * sizeof(float2) : 0);
  p.part_ml_at = take(p.slices > 1 ? BH * p.slices * R * sizeof(float2) : 0);
  p.part_at = take(p.slices > 1 ? BH * p.slices * R * d->d * sizeof(float) : 0);
  p.logits_at = take(keeps_logits(c, p) ? BH * R * p.logits_ld * sizeof(float) : 0);
  p.bytes = at;
  return p;
}

int ig_launch_join(ig_ctx *ctx, const ig_desc *d, const StreamArgs &a, float *mass, hipStream_t stream) {
  const bool logits = mass != nullptr;
  const dim3 block(256);
  const int chunks = logits && d->N ? div_up(d->N, 1024) : 1;
  // four elements a thread where that leaves workgroups for two a compute unit (a chunk of 317 x 4 rows, 32 pools: 38 us
  // with one, 15 with four), one where the trip through memory is what takes the time (13 rows, 32 pools: 4.2 us with
  // four, 3.2 with one; a call for one token over 777 slots 11.0 and 10.3)
  const int E = !logits && (long)d->B * d->H * div_up(a.R, 1024 / d->d) >= 512 ? 4 : 1;
  const int rows = a.slices > 1 ? div_up(a.R, 256 * E / d->d) : 1;
  const FastDiv by_chunks = ig_fast_div(chunks > rows ? chunks : rows), by_threads = ig_fast_div(d->d / E);
  const dim3 jgrid((unsigned)((long)by_chunks.d * d->B * d->H));
#define JOIN_AS(T, E, LOGITS)                                                                        \
  {                                                                                                  \
    auto k = attend_join<T, E, LOGITS>;                                                              \
    IG_LAUNCH(ctx, IG_K_CACHE, k, jgrid, block, stream, a, mass, (int)d->d, by_chunks, by_threads);  \
  }
#define JOIN(T)                                                                                      \
  {                                                                                                  \
    if (logits) JOIN_AS(T, 1, true)                                                                  \
    else if (E == 4) JOIN_AS(T, 4, false)                                                            \
    else JOIN_AS(T, 1, false)                                                                        \
  }
  if (d->dtype == IG_F16) JOIN(half_t) else JOIN(float)
  return IG_OK;
}

int ig_launch_cache(ig_ctx *ctx, const ig_desc *d, const CacheCall &c, const CachePlan &p, char *ws, hipStream_t stream) {
  const bool tree = c.k_tree != nullptr, logits = keeps_logits(c, p);
  const long BH = (long)d->B * d->H;
  StreamArgs a = {};
  a.q = c.q, a.K = c.K, a.V = c.V, a.k_tree = c.k_tree, a.v_tree = c.v_tree, a.out = c.out;
  a.visible = c.visible, a.q_len = c.q_len, a.kv_len = c.kv_len;
  a.n_q = c.n_q, a.R = c.n_q * c.group, a.Hq = d->H * c.group, a.N = d->N, a.N_cap = d->N_cap;
  a.nrb = p.nrb, a.slices = p.slices, a.B = d->B, a.H = d->H;
  a.turn_shift = !p.prompt && d->dtype == IG_F16;
  a.by_slices = ig_fast_div(p.slices), a.by_H = ig_fast_div(d->H), a.by_group = ig_fast_div(c.group);
  a.flip = d->scale < 0.f ? 1 : (d->scale == 0.f ? 2 : 0);
  a.c = (d->scale == 0.f ? 1.f : fabsf(d->scale)) * 1.44269504088896340736f;
  a.stats = c.mass ? reinterpret_cast<float2 *>(ws + p.stats_at) : nullptr;
  a.part_ml = reinterpret_cast<float2 *>(ws + p.part_ml_at);
  a.part = reinterpret_cast<float *>(ws + p.part_at);
  a.logits = reinterpret_cast<float *>(ws + p.logits_at);
  a.logits_ld = p.logits_ld;
  // a causal call with workgroups to spare: each takes a late and an early row block, so that all take equally long
  // (blocks of 128 rows: prompt_rows)
  a.paired = p.prompt && !tree && p.slices == 1 && BH * p.nrb >= 1024 && 2 * c.n_q > d->N;
  const int units = a.paired ? (p.nrb + 1) / 2 : p.nrb;
  a.by_units = ig_fast_div(units), a.by_pair = ig_fast_div(d->B * p.slices * units);
  a.total = (int)(BH * p.slices * units), a.per_xcd = div_up(a.total, 8);
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
    else if constexpr (D <= 128) STREAM(T, D, 2)                                                     \
  }
#define BY_DIM(T, DO)                                                                                \
  switch (d->d) {                                                                                    \
    case 32: DO(T, 32) break;                                                                        \
    case 64: DO(T, 64) break;                                                                        \
    case 128: DO(T, 128) break;                                                                      \
    default: DO(T, 256) break;                                                                       \
  }
#define PROMPT_WAVES(D, NW)                                                                           \
  {                                                                                                  \
    if (tree) {                                                                                      \
      auto k = attend_prompt<D, NW, true>;                                                           \
      IG_LAUNCH(ctx, IG_K_CACHE, k, grid, dim3(NW * 64), stream, a);                                 \
    } else {                                                                                         \
      auto k = attend_prompt<D, NW, false>;                                                          \
      IG_LAUNCH(ctx, IG_K_CACHE, k, grid, dim3(NW * 64), stream, a);                                 \
    }                                                                                                \
  }
#define PROMPT(T, D)                                                                                 \
  {                                                                                                  \
    if constexpr (D == 64 || D == 128) {                                                             \
      if (p.rb == 256) PROMPT_WAVES(D, 8)                                                            \
      else PROMPT_WAVES(D, 4)                                                                        \
    } else                                                                                           \
      PROMPT_WAVES(D, 4)                                                                             \
  }
  if (p.prompt) {
    BY_DIM(half_t, PROMPT)
  } else if (d->dtype == IG_F16) {
    BY_DIM(half_t, STREAM_ROWS)
  } else {
    BY_DIM(float, STREAM_ROWS)
  }
  if (p.slices > 1 || logits)
    if (int rc = ig_launch_join(ctx, d, a, logits ? c.mass : nullptr, stream)) return rc;
  if (!c.mass || logits || d->N == 0) return IG_OK;
  if (d->dtype == IG_F16) {
    // keys in pairs of blocks as the rows above: a prompt's first keys are seen by all of its rows, its last by few
    a.nrb = div_up(d->N, MASS_KEYS);
    a.paired = BH * a.nrb >= 1024 && 2 * c.n_q > d->N;
    const int units = a.paired ? (a.nrb + 1) / 2 : a.nrb;
    a.by_pair = ig_fast_div(units);
    a.total = (int)(BH * units), a.per_xcd = div_up(a.total, 8);
    const dim3 mgrid(a.per_xcd * 8);
#define PROMPT_MASS(T, D)                                                                            \
  {                                                                                                  \
    auto k = prompt_mass<D>;                                                                         \
    IG_LAUNCH(ctx, IG_K_CACHE, k, mgrid, block, stream, a, c.mass);                                  \
  }
    BY_DIM(half_t, PROMPT_MASS)
  } else {
#define MASS(T, D)                                                                                   \
  {                                                                                                  \
    const FastDiv by_chunks = ig_fast_div(div_up(d->N, mass_keys<D>()));                             \
    auto k = attend_mass<D>;                                                                         \
    IG_LAUNCH(ctx, IG_K_CACHE, k, dim3((unsigned)(by_chunks.d * BH)), block, stream, a, c.mass, by_chunks);\
  }
    BY_DIM(float, MASS)
  }
  return IG_OK;
}

// What ig_reserve_cache sizes the workspace for: any number of tokens, slots and slots to keep up to these.  Fewer rows
// or slots can mean more slices, so this is a bound of the parts and not the largest call's plan: a call leaves states
// of at most 64 slices of every row, and of at most ROUNDS rounds of workgroups.
size_t ig_cache_reserve_bytes(const ig_desc *d, int group, int n_q) {
  const long BH = (long)d->B * d->H, R = (long)n_q * group;
  const long rounds = ROUNDS * (d->dtype == IG_F16 ? 256 * slots_of(256) > 128 * slots_of(128) ? 256 * slots_of(256) : 128 * slots_of(128)
                                                   : 32 * slots_of(0));
  const long rows = MOST_SLICES * BH * R < rounds ? MOST_SLICES * BH * R : rounds;
  const size_t logits = group <= 32 ? (size_t)BH * group * (((long)d->N_cap + 63) / 64 * 64) * sizeof(float) : 0;
  const size_t attention = (size_t)BH * R * sizeof(float2) + (size_t)rows * (sizeof(float2) + d->d * sizeof(float)) + logits + 4 * 256;
  ig_desc full = *d;
  full.N = d->N_cap;
  const size_t eviction = ig_evict_workspace(&full, full.N / 2 < 1 ? 1 : full.N / 2);
  return attention > eviction ? attention : eviction;
}
