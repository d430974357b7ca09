// What the kernels over a whole key / value pool share: their arguments, and small device functions.
#pragma once
#include <math.h>

#include "ig_internal.h"

struct StreamArgs {
  const void *q, *K, *V, *k_tree, *v_tree;
  void *out;
  const uint64_t *visible;            // [B][n_q]
  const int32_t *q_len, *kv_len;      // [B], or NULL: n_q, N
  int n_q, R, Hq, N, N_cap;           // R = n_q * group query rows share a pool
  int nrb, slices, total, per_xcd;    // row blocks and slices of a pool, workgroups in all and of one XCD
  int paired;                         // attend_prompt: a workgroup takes two row blocks
  int turn_shift;                     // a workgroup takes 64 << turn_shift slots a turn
  int B, H;
  FastDiv by_pair, by_units;          // workgroups of a head (prompt_mass: of a pool), of a slice
  FastDiv by_slices, by_H, by_group;
  int flip;                           // 1: the scale is negative and q is taken with its sign changed; 2: it is zero, and q is taken as zero
  float c;                            // |scale| / ln 2
  float2 *stats;                      // [B*H][R] reference and 1 / sum of finished rows, or NULL
  float2 *part_ml;                    // [H][B*slices][R] reference and sum of a slice
  float *part;                        // [H][B*slices][R][d]
  float *logits;                      // [B*H][R][logits_ld]
  long logits_ld;
};

// A row's weights are exp2(c s - ref) / sum.  The reference is its largest c s so far, or somewhat less; a row
// that has seen nothing has NOTHING_SEEN, against which every weight is zero, and a sum of zero.
constexpr float NOTHING_SEEN = -1e30f;

// The reference for a largest c s of `top`: `lift` below it where weights are rounded to half precision, whose range above
// one would else lie idle while small weights lose their bits.  Less for logits of 2^20 and more, where the reference's own
// rounding (2^-24 of it) could carry a weight out of that range, and none from 2^22 on.
__device__ __forceinline__ float lifted(float top, float lift) {
  return lift == 0.f ? top : fmaf(-lift, __builtin_amdgcn_fmed3f(fmaf(fabsf(top), -0x1p-22f, 1.f), 0.f, 1.f), top);
}

typedef float floatx16 __attribute__((ext_vector_type(16)));

// Workgroups go to the eight XCDs in turn; this gives every XCD one contiguous run of the work, so that what
// shares keys and values shares an L2.
__device__ __forceinline__ int xcd_order(int id, int per_xcd) { return (id & 7) * per_xcd + (id >> 3); }

// a sequence's length from the caller's array, never outside [0, most]
__device__ __forceinline__ int length_of(const int32_t *len, int b, int all, int most) {
  return len ? min(max(len[b], 0), min(all, most)) : all;
}
// ---- which slices are whose --------------------------------------------------------------------------------
// The B * slices slices of a head are dealt to the sequences by their lengths: one each, and of the others as many as the
// sequence's share of all slots, rounded down, but no more than it has turns of a workgroup and MOST_SLICES at most; what is
// left over stays empty.  (Without lengths from the caller that is `slices` each.)  So a batch of ragged sequences keeps no
// workgroup waiting for the longest one's: one token of 64 sequences of 8192 down to a quarter 270 -> 241 us, a chunk of four
// of 9001 down to a quarter 347 -> 316; what it costs where all are as long is one to two microseconds.
constexpr int MOST_SLICES = 64;
struct Span {
  int b, slice, slices, first;        // the sequence (-1: none), the slice among its own, how many it has, its first one's number
  int kv, nq;                         // its slots and query tokens
};
// the span of slice number `at`, or, BY_SEQUENCE, of sequence `at`
template <bool BY_SEQUENCE> __device__ __forceinline__ Span span_of(const StreamArgs &a, int at) {
  if (a.slices == 1 || !a.kv_len || a.B == 1) {
    const int b = BY_SEQUENCE ? at : a.by_slices.div(at);
    return Span{b, BY_SEQUENCE ? 0 : at - b * a.slices, a.slices, b * a.slices,
                length_of(a.kv_len, b, a.N, a.N_cap), length_of(a.q_len, b, a.n_q, a.n_q)};
  }
  // (the lanes' sequences' lengths in units of 64 slots: B times as many stay below 2^31)
  const int lane = threadIdx.x & 63;
  int kv = length_of(a.kv_len, min(lane, a.B - 1), a.N, a.N_cap), nq = length_of(a.q_len, min(lane, a.B - 1), a.n_q, a.n_q);
  int all = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int len = b0 ? length_of(a.kv_len, min(b0 + lane, a.B - 1), a.N, a.N_cap) : kv;
    all += __builtin_amdgcn_readlane(wave_incl_scan(b0 + lane < a.B ? (len + 63) >> 6 : 0), 63);
  }
  const long spare = (long)a.B * (a.slices - 1);
  const float per_unit = all ? (float)spare / (float)all : 0.f;
  int first = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    if (b0) {
      kv = length_of(a.kv_len, min(b0 + lane, a.B - 1), a.N, a.N_cap);
      nq = length_of(a.q_len, min(b0 + lane, a.B - 1), a.n_q, a.n_q);
    }
    // spare * units / all, rounded down: by float, then put right by the remainder (there are at most some thousand
    // slices, so the float is off by one at most)
    const int units = (kv + 63) >> 6;
    int extra = (int)((float)units * per_unit);
    if ((long)extra * all > spare * units) --extra;
    else if (all && (long)(extra + 1) * all <= spare * units) ++extra;
    // (a slice without slots leaves a state all the same, and the join reads the states eight at a time, one after the other: a
    // token of one sequence of 32768 and 15 of 64 with weights 59 us with 358 slices for the long one, 26 with 64)
    extra = max(0, min(extra, min(MOST_SLICES, (units + a.turn_shift) >> a.turn_shift) - 1));
    const int mine = b0 + lane < a.B ? 1 + extra : 0, incl = wave_incl_scan(mine);
    const int end = first + __builtin_amdgcn_readlane(incl, 63);
    if (BY_SEQUENCE ? at < b0 + 64 : at < end) {
      const int l = BY_SEQUENCE ? at - b0 : __builtin_ctzll(__ballot(first + incl > at));
      const int last = first + __builtin_amdgcn_readlane(incl, l), n = __builtin_amdgcn_readlane(mine, l);
      return Span{b0 + l, BY_SEQUENCE ? 0 : at - (last - n), n, last - n, __builtin_amdgcn_readlane(kv, l), __builtin_amdgcn_readlane(nq, l)};
    }
    first = end;
  }
  return Span{-1, 0, 0, 0, 0, 0};
}

// slots that row `row` of a pool's query rows sees: those of a tree all, those of a prompt up to their own
template <bool TREE> __device__ __forceinline__ int row_limit(const StreamArgs &a, int row, int kv, int nq) {
  return TREE ? kv : max(0, kv - nq + a.by_group.div(row) + 1);
}
__device__ __forceinline__ unsigned long long low_bits(int n) { return n >= 64 ? ~0ull : (1ull << n) - 1; }

// Nodes of a sequence's tree that any node sees (by the whole wave; masks_of, asked for ahead of it, are the lanes'
// nodes').  A node that none sees is never read: its weights are zero, but zero times what it holds need not be.
__device__ __forceinline__ unsigned long long masks_of(const StreamArgs &a, int b, int nq) {
  return a.visible[(long)b * a.n_q + min((int)(threadIdx.x & 63), a.n_q - 1)];
}
__device__ __forceinline__ unsigned long long nodes_seen(unsigned long long masks, int nq) {
  unsigned long long v = (int)(threadIdx.x & 63) < nq ? masks & low_bits(nq) : 0;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v |= __shfl_xor(v, o, 64);
  return (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
         (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
// the node read for node j: itself, or the first one that is seen
__device__ __forceinline__ int node_read(unsigned long long seen, int j) { return seen >> (j & 63) & 1 ? j : __builtin_ctzll(seen); }

// 2^x to the last bit but one; denormal results are zero (a weight of 2^-126 of the largest)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 1 / sum, zero for a row without weights
__device__ __forceinline__ float inverse_of(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

template <typename T> __device__ __forceinline__ uint4 flip_sign(uint4 v, int flip) {
  const unsigned bits = flip == 1 ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u, keep = flip == 2 ? 0u : ~0u;
  return make_uint4((v.x ^ bits) & keep, (v.y ^ bits) & keep, (v.z ^ bits) & keep, (v.w ^ bits) & keep);
}

// 16 bytes of 16 rows of A and 16 columns of B: s += A B over the channels they hold
template <typename T> __device__ __forceinline__ floatx4 dot_step(uint4 a, uint4 b, floatx4 s) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), s, 0, 0, 0);
  } else {
    const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], s, 0, 0, 0);
    return s;
  }
}

// W consecutive words, in loads of up to 16 bytes (the address is aligned to them)
template <int W> __device__ __forceinline__ void load_words(const void *from, unsigned (&to)[W]) {
  if constexpr (W == 1) {
    to[0] = *static_cast<const unsigned *>(from);
  } else if constexpr (W == 2) {
    const uint2 x = *static_cast<const uint2 *>(from);
    to[0] = x.x, to[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const uint4 x = static_cast<const uint4 *>(from)[i];
      to[4 * i] = x.x, to[4 * i + 1] = x.y, to[4 * i + 2] = x.z, to[4 * i + 3] = x.w;
    }
  }
}
template <int W, typename T, int N> __device__ __forceinline__ void store_words(void *to, const T (&from)[N]) {
  static_assert(W * 4 == N * sizeof(T) && W >= 2, "whole words, two or more");
  typedef T vecT __attribute__((ext_vector_type(W == 2 ? 8 / sizeof(T) : 16 / sizeof(T))));
  constexpr int PER = sizeof(vecT) / sizeof(T);
#pragma unroll
  for (int i = 0; i < N / PER; ++i) {
    vecT x;
#pragma unroll
    for (int e = 0; e < PER; ++e) x[e] = from[i * PER + e];
    static_cast<vecT *>(to)[i] = x;
  }
}

// channel j of eight rows that a lane holds as pairs of channels
template <int W> __device__ __forceinline__ half8 column_of(const unsigned (&v)[8][W], int j) {
  uint4 r;
  const unsigned pick = j & 1 ? 0x07060302u : 0x05040100u;
  r.x = __builtin_amdgcn_perm(v[1][j / 2], v[0][j / 2], pick);
  r.y = __builtin_amdgcn_perm(v[3][j / 2], v[2][j / 2], pick);
  r.z = __builtin_amdgcn_perm(v[5][j / 2], v[4][j / 2], pick);
  r.w = __builtin_amdgcn_perm(v[7][j / 2], v[6][j / 2], pick);
  return __builtin_bit_cast(half8, r);
}

// ---- tiles in LDS -----------------------------------------------------------------------------------------
// A tile is rows of D halves with the 16-byte pieces of a row in another order: piece c of row r lies where piece
// c ^ piece_swap(r) would.  16 rows' pieces of one column (what a wave reads of K or Q) and 64 bytes of four
// consecutive rows (of V) then fall on different banks.  The swap of a sum of two rows without common bits is the
// exclusive or of theirs, so a lane's address for rows further on, another half tile or another tile is the same one and
// a constant.
template <int D> __host__ __device__ constexpr int piece_swap(int row) {
  if constexpr (D == 32) return (row >> 2) & 3;
  else if constexpr (D == 64) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
  else return (row & 3) << 2 | ((row >> 2) & 3);
}
// keeps the compiler from working out ahead, and holding, what is made from the value
__device__ __forceinline__ unsigned opaque(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}
// the value is worked out before this point
template <typename V> __device__ __forceinline__ void keep_here(V &v) { asm volatile("" : "+v"(v)); }
typedef const char __attribute__((address_space(3))) *lds_bytes;
__device__ __forceinline__ lds_bytes lds_at(const half_t *tile) {
  return (lds_bytes)(const __attribute__((address_space(3))) half_t *)tile;
}
// Rows of a 32-row block as a product's operand: lane i of either half takes piece 2 k + half of row i.
template <int D> __device__ __forceinline__ unsigned row_offset(int lane, int k) {
  const int i = lane & 31, hb = lane >> 5;
  return i * D * 2 + ((hb ^ piece_swap<D>(i)) * 16 ^ k << 5);
}
__device__ __forceinline__ half8 row_piece(const half_t *rows, unsigned offset) {
  return *reinterpret_cast<const __attribute__((address_space(3))) half8 *>(lds_at(rows) + offset);
}
// Columns of 16 rows (0 .. 3, 8 .. 11 in the lower half wave, 4 .. 7, 12 .. 15 in the upper) as an operand: lane i
// of a half takes column 32 o + i, four rows a call (x = 0: the first four).  The hardware's transposing read takes
// 8 bytes of a row from each of 16 lanes, lane i's from row i / 4, and gives it column i of the four rows.
template <int D> __device__ __forceinline__ unsigned column_offset(int lane, int o, int x) {
  const int i = lane & 15, hb = lane >> 5, r = 4 * hb + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i >> 1) & 1);
  return r * D * 2 + ((c ^ piece_swap<D>(r)) * 16 ^ (o << 6 | x << 5)) + (i & 1) * 8;
}
template <int D> __device__ __forceinline__ uint2 column_rows(const half_t *rows, unsigned offset, int x) {
  typedef __fp16 fp4 __attribute__((__vector_size__(8)));
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4f16((fp4 __attribute__((address_space(3))) *)(
                                       lds_at(rows + 8 * x * D) + offset)));
}
// 64 pieces from memory to LDS without passing through registers: lane i's, `offset` bytes from `from`, to piece i
// of `to` (from and to the same in all lanes).  Not the compiler's builtin, because it waits for every such load
// before any transposing read, also of other LDS; nothing is written but LDS, and who reads it waits
// (wait_for_lds_loads, then a barrier where other waves loaded part of it).
// The compiler does not see what the instruction needs: one wait state after a write of m0, and five after a vector
// instruction (a spilled register's return, say) wrote the address.  The address goes through a scalar move, which is the one
// and for which the hardware itself waits in place of the others.
__device__ __forceinline__ void load_to_lds(const void *from, unsigned offset, half_t *to) {
  const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)to;
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)from), hi = __builtin_amdgcn_readfirstlane((unsigned)((uintptr_t)from >> 32));
  unsigned long long moved;
  asm volatile("s_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(moved) : "{m0}"(__builtin_amdgcn_readfirstlane(at)), "v"(offset),
               "s"((unsigned long long)hi << 32 | lo) : "memory");
}
template <int LEFT> __device__ __forceinline__ void wait_for_lds_loads() {      // all but the newest LEFT
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}

// Between lanes of one wave that write LDS and others of it that read there (or the other way round): a wave's accesses to
// LDS are done in their order, so nothing waits, but the compiler must not change that order.
__device__ __forceinline__ void lanes_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// the other half wave's value and this one's: both in both
__device__ __forceinline__ float both_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// over the four lanes that hold a column of a 16x16 product: l, l + 16, l + 32, l + 48
__device__ __forceinline__ float column_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return both_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float column_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return both_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
