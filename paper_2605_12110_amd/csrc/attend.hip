// Dense attention of new rows over the paged cache (absb_attend_rows, absb_attend_shared).
//
// Every row sees an interval of keys: causal order, window, documents, prefixes and shared prefixes all bound it from below or
// above.  A tile of rows (token, query head of one KV head's group) goes over the keys of its rows' intervals block by block with
// the running maximum and sum of a softmax; blocks that all rows see need no mask, blocks that none sees are not read.
//
//   S^T = K Q^T  32 keys x 32 rows in a 32x32x16 product: a lane then holds 16 scores of ONE row (row = lane % 32), so
//                maxima and sums are a lane's own but for one exchange with lane ^ 32, and a row's factors need no
//                broadcast;
//   O^T += V^T P^T  32 channels x 32 rows: with the keys taken in the order in which the lanes hold them, S^T's registers,
//                rounded in pairs, are the operand P^T as they stand.  V^T comes from row-major V by the transposing read.
//
// Wide tiles, 128 rows: four waves of 32 go over the same keys, 64 at a time, so a key is read once for 128 rows; bound by the matrix
// unit (32 query and 8 KV heads, f16: a prompt of 4 K 153 us, 895 TFLOP/s; 16 K 2180, 1010; a chunk of 1 K behind 32 K 970) at
// a clock that power holds at 1.65 GHz.  Of 256 registers a lane, kernels with a cap and a bias spill 2, with a wide cap 6, with
// that and a bias 4.  Two work-groups a compute unit: with one, 875 TFLOP/s at 16 K instead of 1036.
// Narrow ones, 32 rows: four waves with keys of their own, none waiting for another; bound by memory (a token behind
// 128 K 88 us, 6.1 TB/s).
//
// K and V are copied from their pages straight to LDS, a block ahead, 16 bytes a lane.  The copy writes lanes side by side, so
// what spreads a read over the banks is which piece of a row a lane fetches: K's piece p of row r lies at p ^ (r % 16), V's at
// p ^ 4 (r % 4).
#include <algorithm>
#include <type_traits>

#include "attend.h"

namespace absb {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int ATT_THREADS = 256, ATT_WAVES = 4;
constexpr int LEAST_KEYS = 256;  // of a split, if it is planned to have as many
constexpr int ROW_BYTES = ABSB_HEAD_DIM * 2;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <int DT>
__device__ __forceinline__ f32x16 mma_32x32x16(u32x4 a, u32x4 b, f32x16 c) {
  if (DT == ABSB_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(bitcast<half8_t>(a), bitcast<half8_t>(b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(bitcast<bf16x8_t>(a), bitcast<bf16x8_t>(b), c, 0, 0, 0);
}

// Two values rounded to the K/V type, side by side.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if (DT == ABSB_F16) {
    half2_t h = {(_Float16)a, (_Float16)b};
    return bitcast<uint32_t>(h);
  }
  bf16x2_t h = {(__bf16)a, (__bf16)b};
  return bitcast<uint32_t>(h);
}

// The other half of the wave's value.
template <typename Op>
__device__ __forceinline__ float across_halves(float x, Op op) {
  const auto h = __builtin_amdgcn_permlane32_swap(bitcast<uint32_t>(x), bitcast<uint32_t>(x), false, false);
  return op(bitcast<float>(h[0]), bitcast<float>(h[1]));
}

// The owner of tile slot x, its rows [row0(o), row0(o + 1)), its first slot.  Few owners: by a sum over their tiles.  Many: the largest
// o in [0, n) with slot0(o) <= x, where slot0(o) = row0(o) * G / tile + o; the wave looks at 64 places at a time.
struct Owner {
  int o, r0, r1, len;  // ... and lens[o]
  int64_t slot0;
};
template <typename F>
__device__ __forceinline__ Owner owner_of(int n, int64_t x, int G, int log2_tile, const int32_t* lens, F row0) {
  const int lane = threadIdx.x & 63;
  if (n <= DENSE_OWNERS) {
    const int r = row0(min(lane, n)), len = lens[min(lane, n - 1)];
    const int next = __shfl(r, min(lane + 1, 63));
    const uint32_t tiles = ((uint32_t)(next - r) * (uint32_t)G + (1u << log2_tile) - 1) >> log2_tile;
    uint32_t total;
    const uint32_t before = wave_incl_scan_u32(lane < n ? tiles : 0, &total) - (lane < n ? tiles : 0);
    const int i = max(0, __popcll(__ballot(lane < n && (int64_t)before <= x)) - 1);
    return Owner{i, __builtin_amdgcn_readlane(r, i), __builtin_amdgcn_readlane(r, i + 1), __builtin_amdgcn_readlane(len, i),
                 __builtin_amdgcn_readlane((int)before, i)};
  }
  int lo = 0, hi = n;  // the owner is in [lo, hi)
  while (hi - lo > 63) {
    const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
    const uint64_t below = __ballot(at < hi && (((int64_t)row0(min(at, hi - 1)) * G) >> log2_tile) + at <= x);
    lo += max(0, __popcll(below) - 1) * step;
    hi = min(hi, lo + step);
  }
  const int at = min(lo + lane, hi), r = row0(at), len = lens[min(at, n - 1)];
  const uint64_t below = __ballot(lo + lane < hi && (((int64_t)r * G) >> log2_tile) + at <= x);
  const int i = max(0, __popcll(below) - 1);
  const int r0 = __builtin_amdgcn_readlane(r, i);
  return Owner{lo + i, r0, __builtin_amdgcn_readlane(r, i + 1), __builtin_amdgcn_readlane(len, i), (((int64_t)r0 * G) >> log2_tile) + lo + i};
}
// The shared tokens of request b: those of the last group g with first[g] <= b.  `first`, `len`: the lane's group of the first 64,
// asked for beforehand.
__device__ __forceinline__ int shared_tokens(const AttendParams& p, int b, int first, int len) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = p.groups;
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
    lo += max(0, __popcll(__ballot(at < hi && p.first[min(at, hi - 1)] <= b)) - 1) * step;
    hi = min(hi, lo + step);
    if (hi - lo <= 64) {
      const int mine = min(lo + lane, hi - 1);
      first = p.first[mine];
      len = p.len[mine];
    }
  }
  return __builtin_amdgcn_readlane(len, max(0, __popcll(__ballot(lo + lane < hi && first <= b)) - 1));
}

struct RowOf {
  int row, head;       // row of q and out, query head; row < 0: none
  int pos, lo, hi;     // position, first and last key seen
};

// What a work-group's tile is about.
struct Tile {
  int table_row, limit;     // whose page-table row; keys it holds
  int r0, n;                // the owner's first row, rows (tokens)
  int tok0, g0;             // the tile's first (token, head) pair
  int pairs;                // of the owner from there on
};

// Softmax state and output of a wave's 32 rows: lane l holds row l % 32; O[t][i] is channel 32 t + 8 (i / 4) + 4 (l / 32) + i % 4.
// Two sums of weights: `l` as rounded for the product with V, by which the output is divided (it stays a convex combination of
// value rows: with one dominant key, or many equal ones, all of the mass rounds the same way, and an output divided by the
// other sum would be off by up to 2^-8 in bf16); `lx` before rounding, of which the log-sum is made.
struct State {
  float m, l, lx;
  f32x16 o[4];
};

// Scores q.k in log2 units: the cap, then the distance bias (`away`: from the row to the key).  CAP_WIDE: a cap so far above
// ordinary scores that small ones need another form, whose error is in proportion to the score.
enum : int { CAP_NONE = 0, CAP_PLAIN = 1, CAP_WIDE = 2 };
template <int CAP, bool BIAS>
__device__ __forceinline__ float score_of(const AttendParams& p, float s, float slope_log2, float away) {
  float x = s;
  if (CAP) {
    // cap tanh(y) = cap - 2 cap / (e^2y + 1).  The exponential and the reciprocal are good to 2^-23 of themselves, the sum to 2^-24:
    // off by 2 * 2^-23 cap around y = 0, by 3 * 2^-23 cap at most (where tanh is near -1) ...
    const float u = s * p.cap_in;  // 2 y log2(e)
    x = __builtin_fmaf(-2.0f * p.cap_log2, __builtin_amdgcn_rcpf(exp2_fast(u) + 1.0f), p.cap_log2);
    if (CAP == CAP_WIDE) {  // ... that is by 10 * 2^-23 of the result where |y| >= 1/4; for smaller ones, the series
      const float y = u * (0.5f * LN2), z = y * y;
      const float series = y * (1.0f + z * (-1.0f / 3 + z * (2.0f / 15 + z * (-17.0f / 315 + z * (62.0f / 2835)))));
      x = __builtin_fabsf(y) < 0.25f ? series * p.cap_log2 : x;
    }
  }
  if (BIAS) x = __builtin_fmaf(-slope_log2, __builtin_fabsf(away), CAP ? x : x * p.scale_log2);
  return x;
}
// Keeps the compiler from making a branch that hardly any block takes into selects that every block pays for.
__device__ __forceinline__ void rarely() { asm volatile(""); }

// S^T of the 32 keys whose K rows are at `kl`: score i of a lane is of key 8 (i / 4) + 4 half + i % 4.  (Two chains of products: a
// lone wave waits for each of a chain.)
template <int DT>
__device__ __forceinline__ f32x16 scores_of(const char* kl, const u32x4 (&q)[8]) {
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  f32x16 s[2] = {};
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(kl + col * ROW_BYTES + (((2 * c + half) ^ (col & 15)) * 16));
    s[c & 1] = mma_32x32x16<DT>(a, q[c], s[c & 1]);
  }
  return s[0] + s[1];
}

// How far a row is from key 0 of a lane's scores of the 32 keys from k0 on.  (Exact below 2^24 tokens; beyond, off by a part in 2^24.)
__device__ __forceinline__ float away_from(const RowOf& row, int k0) {
  return (float)(row.pos - (k0 + 4 * (int)((threadIdx.x & 63) >> 5)));
}
constexpr int key_of(int i) { return 8 * (i >> 2) + (i & 3); }  // score i of a lane's 16: which key behind the lane's first
// -inf where a row does not see a key of the 32 KT from k0 on.
template <int KT>
__device__ __forceinline__ void hide(f32x16 (&s)[KT], int k0, const RowOf& row) {
  const int first_key = k0 + 4 * (int)((threadIdx.x & 63) >> 5), lo = row.lo - first_key, hi = row.hi - first_key;
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = 32 * t + key_of(i);
      s[t][i] = at >= lo && at <= hi ? s[t][i] : -__builtin_inff();
    }
}
template <int CAP, bool BIAS, int KT>
__device__ __forceinline__ void adjust(const AttendParams& p, f32x16 (&s)[KT], int k0, const RowOf& row, float slope_log2) {
  const float away = BIAS ? away_from(row, k0) : 0.0f;
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[t][i] = score_of<CAP, BIAS>(p, s[t][i], slope_log2, away - (float)(32 * t + key_of(i)));
}

// The maximum that the rows' weights are taken against.  It follows the scores' own only when they exceed it by 2^RISE:
// weights then reach 2^RISE, which the K/V types hold to the same relative step as those below 1 (and the output is divided by
// their sum as rounded), and the output is hardly ever scaled again (with the true maximum some of a wave's 32 rows has a new
// one in most blocks).
constexpr float RISE = 8.0f;
template <int KT>
__device__ __forceinline__ float largest(const f32x16 (&s)[KT]) {
  float mx = -__builtin_inff();
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[t][i]);
  return mx;
}
template <bool SCALED>
__device__ __forceinline__ float new_maximum(const AttendParams& p, float mx, State& st) {
  mx = across_halves(mx, [](float a, float b) { return fmaxf(a, b); });
  if (!SCALED) mx *= p.scale_log2;
  const bool rises = mx > st.m + RISE;  // (the first key seen: above -inf)
  if (__any(rises)) {
    rarely();
    const float mn = rises ? mx : st.m;
    const float alpha = rises ? exp2_fast(st.m - mn) : 1.0f;
    const bool some = __any(st.m != -__builtin_inff());  // (else the output is still zero)
    st.m = mn;
    st.l *= alpha;
    st.lx *= alpha;
    if (some) {
#pragma unroll
      for (int t = 0; t < 4; ++t) st.o[t] *= alpha;
    }
  }
  return st.m == -__builtin_inff() ? 0.0f : st.m;  // nothing seen yet: weights 0, not NaN
}

// Two rounded weights onto a sum in binary32.
template <int DT>
__device__ __forceinline__ float add_pair(uint32_t w, float sum) {
  return Elem<DT>::dot2(w, DT == ABSB_F16 ? 0x3c003c00u : 0x3f803f80u, sum);
}

// Weights of the scores, rounded to the K/V type (two to a word: P^T as the product takes it), and their sums.
template <int DT, bool SCALED, int KT>
__device__ __forceinline__ void weigh(const AttendParams& p, const f32x16 (&s)[KT], float base, u32x4 (&w)[2 * KT], State& st) {
  float sum = 0.0f, rounded = 0.0f;
#pragma unroll
  for (int c = 0; c < 2 * KT; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = s[c >> 1][8 * (c & 1) + 2 * j], b = s[c >> 1][8 * (c & 1) + 2 * j + 1];
      const float x = exp2_fast(SCALED ? a - base : __builtin_fmaf(a, p.scale_log2, -base));
      const float y = exp2_fast(SCALED ? b - base : __builtin_fmaf(b, p.scale_log2, -base));
      sum += x;
      sum += y;
      w[c][j] = pack2<DT>(x, y);
      rounded = add_pair<DT>(w[c][j], rounded);
    }
  st.l += rounded;
  st.lx += sum;
}

// O^T += V^T P^T for the 32 KT keys whose V rows are at `vl`.
template <int DT, int KT>
__device__ __forceinline__ void add_values(const char* vl, const u32x4 (&w)[2 * KT], State& st) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
  for (int c = 0; c < 2 * KT; ++c) {
    // V^T: of 16 lanes, lane i points at channels 4 (i % 4).. of key i / 4 and gets channel i of the four keys
    const int i16 = lane & 15, grp = (lane >> 4) & 1, key = 16 * c + 4 * half + (i16 >> 2);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int piece = (4 * t + 2 * grp + ((i16 & 3) >> 1)) ^ ((key & 3) << 2);
      const char* at = vl + key * ROW_BYTES + piece * 16 + (i16 & 1) * 8;
      typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
      const u32x2 lo = bitcast<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at)));
      const u32x2 hi = bitcast<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 8 * ROW_BYTES)));
      st.o[t] = mma_32x32x16<DT>(u32x4{lo[0], lo[1], hi[0], hi[1]}, w[c], st.o[t]);
    }
  }
}

// The main part of a step of a wide tile, in an order of its own (the compiler's would wait for every read of LDS right before its
// product): 16 products of the next block's scores, then 16 of this block's weights with its values; beside each, the vector work
// of one score or two, and the read that the fourth product after it needs.  A product takes the matrix unit 32 cycles, an
// exponential the vector unit 16, its other work 12 and half an instruction of the rounded sum (which cost 3 % of a 4096-token prompt).  `mx`: the largest of a lane's next scores; `away`: of the row from their
// first key.
template <int DT, int CAP, bool BIAS>
__device__ __forceinline__ void wide_step(const AttendParams& p, const char* kl, const char* vl, const u32x4 (&q)[8], const f32x16 (&s)[2],
                                          float base, f32x16 (&s_next)[2], float& mx, State& st, float slope_log2, float away) {
  constexpr bool SCALED = CAP || BIAS;  // (else the scores are still q.k)
  constexpr int AHEAD = 4, SLOTS = 32;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5, i16 = lane & 15, grp = (lane >> 4) & 1;
  u32x4 f[AHEAD], w[4];
  float x = 0.0f, sum = 0.0f, rounded = 0.0f;
  mx = -__builtin_inff();
  auto fetch = [&](int j) __attribute__((always_inline)) {  // the operand of product j
    if (j < 16) {
      const int t = j & 1, c = j >> 1;
      f[j % AHEAD] = *reinterpret_cast<const u32x4*>(kl + (32 * t + col) * ROW_BYTES + (((2 * c + half) ^ (col & 15)) * 16));
    } else {
      // V^T: of 16 lanes, lane i points at channels 4 (i % 4).. of key i / 4 and gets channel i of the four keys
      const int c = (j - 16) >> 2, t = j & 3, key = 16 * c + 4 * half + (i16 >> 2);
      const int piece = (4 * t + 2 * grp + ((i16 & 3) >> 1)) ^ ((key & 3) << 2);
      const char* at = vl + key * ROW_BYTES + piece * 16 + (i16 & 1) * 8;
      typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
      const u32x2 lo = bitcast<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at)));
      const u32x2 hi = bitcast<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 8 * ROW_BYTES)));
      f[j % AHEAD] = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  };
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) fetch(j);
  const f32x16 zero = {};
  __builtin_amdgcn_s_setprio(1);  // (the other wave of a SIMD then falls out of step: 4096-token prompt 156 -> 152 us)
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    if (j < 16)
      s_next[j & 1] = mma_32x32x16<DT>(f[j % AHEAD], q[j >> 1], j < 2 ? zero : s_next[j & 1]);
    else
      st.o[j & 3] = mma_32x32x16<DT>(f[j % AHEAD], w[(j - 16) >> 2], st.o[j & 3]);
    if (j + AHEAD < SLOTS) fetch(j + AHEAD);
    // 32 weights in 28 slots: those of 16 keys are there before their product
#pragma unroll
    for (int e = j * 8 / 7; e < (j + 1) * 8 / 7 && e < 32; ++e) {
      const float a = s[e >> 4][e & 15];
      const float y = exp2_fast(SCALED ? a - base : __builtin_fmaf(a, p.scale_log2, -base));
      sum += y;
      if (e & 1) {
        w[e >> 3][(e & 7) >> 1] = pack2<DT>(x, y);
        rounded = add_pair<DT>(w[e >> 3][(e & 7) >> 1], rounded);
      } else {
        x = y;
      }
    }
    // the next scores, which the sixteenth product has completed: what the softmax takes, and their maximum
    if (j >= 18) {
#pragma unroll
      for (int e = (j - 18) * 16 / 7; e < (j - 17) * 16 / 7; ++e) {
        float y = s_next[e >> 4][e & 15];
        if (SCALED) y = score_of<CAP, BIAS>(p, y, slope_log2, away - (float)(32 * (e >> 4) + key_of(e & 15)));
        s_next[e >> 4][e & 15] = y;
        mx = fmaxf(mx, y);
      }
    }
    asm volatile("" : "+v"(sum), "+v"(rounded));  // (the sums are made here, not out of 32 kept values at the end)
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  st.l += rounded;
  st.lx += sum;
}

__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) |
         ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32);
}

// Where the rows of 512 keys lie: lane j of the wave has the byte offset of keys 8 j .. 8 j + 7 of the stretch (they share a
// page) and which of the eight is the last that exists.  In two halves: the page is asked for a stretch ahead, and the
// offset worked out when the stretch begins.
struct Stretch {
  uint64_t off;
  int most;
};
__device__ __forceinline__ int first_of_lane(int k0, int limit) {
  return (int)min((int64_t)k0 + 8 * (threadIdx.x & 63), (int64_t)limit - 1) & ~7;
}
__device__ __forceinline__ int32_t ask_page(const AttendParams& p, const int32_t* pages, int k0, int limit) {
  return pages[first_of_lane(k0, limit) >> p.log2_page];
}
__device__ __forceinline__ Stretch stretch_on(const AttendParams& p, int32_t page, int k0, int limit) {
  const int at = first_of_lane(k0, limit);
  Stretch s;
  s.off = (uint64_t)page * (uint64_t)p.s_page + (uint64_t)(at & ((1 << p.log2_page) - 1)) * (uint64_t)p.s_tok;
  s.most = min(7, limit - 1 - at);
  return s;
}

// 16 bytes a lane from `base` (+ a lane's 32-bit offset) to LDS, lanes side by side from `to` on.  As the instruction itself: the
// compiler would wait for every copy in flight ahead of every read of LDS, the one of the next block included.  (It must wait
// for none: copies_done() does, in front of the barrier behind which a block is read.  The waits: m0 wants one state ahead of the
// copy, a scalar that came from a vector instruction five.)
// (m0 is nobody's register, which the compiler warns of; that the copy changes it is said all the same, should it come to use it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool STREAM>  // past the caches
__device__ __forceinline__ void copy_to_lds(const char* base, uint32_t lane_off, uint32_t to) {
  if (STREAM)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(to), "v"(lane_off), "s"(base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(lane_off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const char* at) {
  typedef __attribute__((address_space(3))) const char* lds;
  return (uint32_t)(uintptr_t)(lds)(at);
}

// What copies of rows need of a lane: it fetches piece lane % 16 (of 16 bytes) of row lane / 16 of four, so that lanes side by
// side in LDS hold what lies at p ^ (r % 16) of K's row r, at p ^ 4 (r % 4) of V's.
struct LaneCopy {
  uint32_t key[4], value[2];  // byte offsets from eight keys' first row: of K's rows 4 i .. 4 i + 3 of 16, of V's (upper four: 1)
};
__device__ __forceinline__ LaneCopy lane_copy(uint32_t pitch) {
  const uint32_t lane = threadIdx.x & 63, piece = lane & 15, r4 = lane >> 4;
  LaneCopy c;
#pragma unroll
  for (int i = 0; i < 4; ++i) c.key[i] = (4 * (i & 1) + r4) * pitch + ((piece ^ (4 * i + r4)) * 16);
#pragma unroll
  for (int i = 0; i < 2; ++i) c.value[i] = (4 * i + r4) * pitch + ((piece ^ (r4 << 2)) * 16);
  return c;
}
// N times eight rows of a block: where they start, the last of each that exists, and whether all do.
template <int N>
struct Groups {
  uint64_t off[N];
  int most[N];
  bool full;
};
// Copies them from K or V to LDS, 2 N copies; rows that do not exist are the last that does again, which no one sees.
template <bool KEY, bool STREAM, int N>
__device__ __forceinline__ void copy_groups(const char* base, const Groups<N>& g, uint32_t pitch, const LaneCopy& lc, uint32_t to) {
  auto copy = [&](auto all) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2 * N; ++j) {
      uint32_t at = KEY ? lc.key[j & 3] : lc.value[j & 1];
      if (!decltype(all)::value) at -= (uint32_t)max(0, 4 * (j & 1) + (int)((threadIdx.x & 63) >> 4) - g.most[j >> 1]) * pitch;
      copy_to_lds<STREAM>(base + g.off[j >> 1], at, to + 4 * j * ROW_BYTES);
    }
  };
  if (g.full) {
    copy(std::true_type());
  } else {
    rarely();
    copy(std::false_type());
  }
}

// The wave's copies have arrived, and what it read of LDS has, too (the next copy may overwrite it).
__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
// All but the last N loads of the wave have arrived (they do in order).
template <int N>
__device__ __forceinline__ void copies_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// What the wave read of LDS has arrived: a copy may take its place.
__device__ __forceinline__ void lds_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Which (token, query head of the group) pair i of a tile is: a division by the group size that a product does for i < 8192.
struct PairOf {
  int tok, g;
};
__device__ __forceinline__ PairOf pair_of_tile(const AttendParams& p, const Tile& t, int i) {
  const int x = t.g0 + i, tok = (x * p.inv_G) >> 16;
  return PairOf{t.tok0 + tok, x - tok * p.G};
}
// Pair i of a tile, and the interval of keys that it sees.
__device__ __forceinline__ RowOf row_of(const AttendParams& p, const Tile& t, bool shared, int own_from, int group, int kv_head, int i) {
  RowOf r;
  r.row = -1;
  r.head = kv_head * p.G;
  r.pos = 0;
  r.lo = 0;
  r.hi = -1;
  if (i >= t.pairs) return r;
  const PairOf pair = pair_of_tile(p, t, i);
  const int tok = pair.tok;
  r.row = t.r0 + tok;
  r.head += pair.g;
  const int b = t.table_row;
  if (shared) {
    r.hi = t.limit - 1;
    if (p.window || p.slopes) {  // the request that the row belongs to
      int lo = p.first[group], hi = p.first[group + 1];
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.row_off[mid] <= r.row) lo = mid; else hi = mid;
      }
      r.pos = p.seq_lens[lo] - (p.row_off[lo + 1] - r.row);
    }
  } else {
    r.pos = t.limit - t.n + tok;
    r.hi = r.pos;
    if (p.prefix_lens) r.hi = min(max(r.hi, p.prefix_lens[b] - 1), t.limit - 1);
    r.lo = own_from;
  }
  if (p.window) r.lo = max(r.lo, r.pos - p.window + 1);
  if (p.doc_start) r.lo = max(r.lo, p.doc_start[r.row]);
  return r;
}

// Wide: a block of 64 keys, twice.  Narrow: 32 keys a wave, and later the waves' outputs, whose rows lie four banks apart.
constexpr int NARROW_PITCH = ABSB_HEAD_DIM + 4, ATT_LDS = ATT_WAVES * 32 * NARROW_PITCH * 4;
static_assert(ATT_LDS >= 65536 && 2 * (ATT_LDS + 2048) <= 160 * 1024, "two work-groups a compute unit");

template <int DT, int CAP, bool BIAS>
__global__ __launch_bounds__(ATT_THREADS, 2) void attend_kernel(AttendParams p) {
  __shared__ __align__(16) char s_kv[ATT_LDS];
  __shared__ float s_ml[ATT_WAVES][3][32];
  __shared__ int s_lo[ATT_WAVES], s_hi[ATT_WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  fetch_arguments<0, sizeof(AttendParams)>();  // (what follows is a chain of round trips; the arguments make one of it)

  // ---- which phase, tile, KV head and split: heads go round the dies first, so that a head's keys stay in one die's L2 where
  // there are eight; long tiles (prefixes, the last ones of a causal prompt) start first
  const bool shared = blockIdx.x < p.shared_units;
  const uint32_t unit = shared ? blockIdx.x : blockIdx.x - p.shared_units;
  const AttendPhase& ph = shared ? p.shared : p.own;
  const int owners = ph.owners, splits = ph.splits, log2_tile = ph.log2_tile;
  const bool stream = ph.stream;
  const int part0 = shared ? 0 : p.shared.splits;
  const bool wide = log2_tile == 7;
  const int kv_head = (int)(unit % (uint32_t)p.Hkv);
  const uint32_t rest = unit / (uint32_t)p.Hkv;
  const bool cut = (int64_t)rest >= ph.whole;
  const uint32_t among = cut ? rest - (uint32_t)ph.whole : 0;
  const int split = (int)(among % (uint32_t)splits);
  const int64_t slot = ph.slots - 1 - (cut ? ph.whole + (int64_t)(among / (uint32_t)splits) : (int64_t)rest);
  int group_first = 0, group_len = 0;
  if (!shared && p.groups) {
    const int mine = min(lane, p.groups - 1);
    group_first = p.first[mine];
    group_len = p.len[mine];
  }
  const Owner own = owner_of(owners, slot, p.G, log2_tile, shared ? p.len : p.seq_lens, [&](int o) { return p.row_off[shared ? p.first[o] : o]; });
  const int owner = own.o;
  Tile t;
  t.r0 = own.r0;
  t.n = own.r1 - own.r0;
  // (an owner's pairs are fewer than 2^31: absb_attend_* sees to it)
  const uint32_t f0 = (uint32_t)(slot - own.slot0) << log2_tile;
  t.pairs = (int)((uint32_t)t.n * (uint32_t)p.G - f0);
  if (t.pairs <= 0) return;
  t.tok0 = (int)(f0 / (uint32_t)p.G);
  t.g0 = (int)(f0 - (uint32_t)t.tok0 * p.G);
  t.table_row = shared ? p.first[owner] : owner;
  t.limit = own.len;
  const int own_from = !shared && p.groups ? shared_tokens(p, owner, group_first, group_len) : 0;

  const RowOf row = row_of(p, t, shared, own_from, owner, kv_head, (wide ? 32 * wave : 0) + (lane & 31));
  const bool valid = row.row >= 0;
  // (asked for ahead of what the keys wait for: tiles of a few keys 63.6 -> 61.0 us of 2560, 12.2 -> 11.8 us of a small step)
  u32x4 q[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    q[c] = u32x4{0u, 0u, 0u, 0u};
    if (valid) q[c] = *reinterpret_cast<const u32x4*>(p.q + ((int64_t)row.row * p.Hq + row.head) * ABSB_HEAD_DIM + (2 * c + (lane >> 5)) * 8);
  }
  const bool sees = valid && row.lo <= row.hi;
  const int lo = sees ? row.lo : INT32_MAX, hi = sees ? row.hi : -1;
  auto lesser = [](uint32_t a, uint32_t b) { return a < b ? a : b; };
  auto greater = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  const int wave_lo = (int)wave_reduce_u32((uint32_t)lo, lesser), wave_hi = (int)wave_reduce_u32((uint32_t)(hi + 1), greater) - 1;
  // keys that every row of the wave sees (rows that do not exist see whatever the others do)
  const int all_lo = (int)wave_reduce_u32((uint32_t)(valid ? row.lo : 0), greater);
  const int all_hi = (int)wave_reduce_u32((uint32_t)((valid ? row.hi : INT32_MAX - 1) + 1), lesser) - 1;
  int tile_lo = wave_lo, tile_hi = wave_hi;
  if (wide) {
    if (lane == 0) {
      s_lo[wave] = wave_lo;
      s_hi[wave] = wave_hi;
    }
    __syncthreads();
    tile_lo = min(min(s_lo[0], s_lo[1]), min(s_lo[2], s_lo[3]));
    tile_hi = max(max(s_hi[0], s_hi[1]), max(s_hi[2], s_hi[3]));
  }
  State st;
  st.m = -__builtin_inff();
  st.l = st.lx = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) st.o[i][j] = 0.0f;

  // ---- the split's keys [begin, end)
  // The tile's keys are divided evenly: windows and documents leave it fewer than the host has planned for, and some requests are short
  // (twice 32 tokens of documents of 1900 behind 34 K: 44 us in stretches as planned, 18.6; 8 tokens behind 4 to 32 K 107, 104).
  const int first = tile_lo & ~63;
  const uint32_t keys = tile_lo <= tile_hi ? (uint32_t)(tile_hi + 1 - first) : 0;
  const int64_t chunk = cut ? max(min((uint32_t)LEAST_KEYS, (uint32_t)ph.chunk), ((keys + splits - 1) / (uint32_t)splits + 127) & ~127u) : int64_t(1) << 31;
  const int64_t from = (int64_t)first + split * chunk;
  const int begin = (int)min(from, (int64_t)tile_hi + 1);
  const int end = (int)min(from + chunk, (int64_t)tile_hi + 1);
  if (begin < end) {
    const float slope_log2 = BIAS && valid ? p.slopes[row.head] * LOG2E : 0.0f;
    const int32_t* pages = p.page_table + (int64_t)t.table_row * p.pt_stride;
    const char *kb = p.k + kv_head * p.s_head, *vb = p.v + kv_head * p.s_head;
    constexpr bool SCALED = CAP || BIAS;
    auto stretch_begin = [&](int n) { return (int)min((int64_t)begin + (int64_t)n * 512, (int64_t)t.limit - 1); };
    auto ask = [&](int n) { return ask_page(p, pages, stretch_begin(n), t.limit); };
    auto stretch = [&](int n, int32_t page) { return stretch_on(p, page, stretch_begin(n), t.limit); };
    const uint32_t pitch = (uint32_t)p.s_tok;  // (seven rows of at most 2^29 bytes)
    const LaneCopy lc = lane_copy(pitch);
    // This wave's N groups of eight rows of a block: from lane `from` of the stretch on.
    auto groups = [&](const Stretch& s, int from, auto n) __attribute__((always_inline)) {
      Groups<decltype(n)::value> g;
      g.full = true;
#pragma unroll
      for (int j = 0; j < decltype(n)::value; ++j) {
        g.off[j] = lane_u64(s.off, from + j);
        g.most[j] = __builtin_amdgcn_readlane(s.most, from + j);
        g.full = g.full && g.most[j] == 7;
      }
      return g;
    };
    Stretch at = stretch(0, ask(0));
    int32_t next = ask(1);
    auto wide_tile = [&](auto past) __attribute__((always_inline)) {
      constexpr bool STREAM = decltype(past)::value;
      constexpr int STEP = 64, PER = 512 / STEP, STAGE = STEP * ROW_BYTES;
      const int steps = (end - begin + STEP - 1) / STEP;
      const char* mine = s_kv;
      const uint32_t to = lds_address(s_kv) + 16 * wave * ROW_BYTES;
      auto copy_k = [&](const Groups<2>& g, int i) __attribute__((always_inline)) { copy_groups<true, STREAM>(kb, g, pitch, lc, to + (i & 1) * STAGE); };
      auto copy_v = [&](const Groups<2>& g, int i) __attribute__((always_inline)) { copy_groups<false, STREAM>(vb, g, pitch, lc, to + (2 + (i & 1)) * STAGE); };
      auto rows_of = [&](int i) __attribute__((always_inline)) { return groups(at, (i % PER) * 8 + 2 * wave, std::integral_constant<int, 2>()); };
      Groups<2> rows = rows_of(0);
      // Step i: the scores of block i + 1 are worked out beside the softmax of block i, matrix and vector unit at once; so K is
      // copied two blocks ahead, V one.  (The last step works out scores of whatever is in LDS, for nobody.)
      copy_k(rows, 0);
      copy_v(rows, 0);
      copies_done();
      __syncthreads();
      rows = rows_of(1);
      if (steps > 1) copy_k(rows, 1);
      const bool live = wave_lo <= wave_hi;  // (waves whose rows see nothing only copy)
      f32x16 s0[2], s1[2];
      if (live) {
        s0[0] = scores_of<DT>(mine, q);
        s0[1] = scores_of<DT>(mine + 32 * ROW_BYTES, q);
      }
      if (SCALED) adjust<CAP, BIAS, 2>(p, s0, begin, row, slope_log2);
      float mx = live ? largest<2>(s0) : 0.0f;
      auto step = [&](int i, f32x16 (&s)[2], f32x16 (&s_next)[2]) __attribute__((always_inline)) {
        const char *kl = mine + ((i + 1) & 1) * STAGE, *vl = mine + 2 * STAGE + (i & 1) * STAGE;
        copies_done();
        __syncthreads();  // K of block i + 1 and V of block i are there, and nobody reads the ones before any more
        if (i + 1 < steps) copy_v(rows, i + 1);
        if (i + 2 < steps) {
          if ((i + 2) % PER == 0) {
            at = stretch((i + 2) / PER, next);
            next = ask((i + 2) / PER + 1);
          }
          rows = rows_of(i + 2);
          copy_k(rows, i + 2);
        }
        if (!live) return;
        const int k0 = begin + i * STEP;
        if (k0 < all_lo || k0 + 63 > all_hi) {
          rarely();
          hide<2>(s, k0, row);
          mx = largest<2>(s);
        }
        const float base = new_maximum<SCALED>(p, mx, st);
        wide_step<DT, CAP, BIAS>(p, kl, vl, q, s, base, s_next, mx, st, slope_log2, BIAS ? away_from(row, k0 + STEP) : 0.0f);
      };
      for (int i = 0; i < steps; i += 2) {
        step(i, s0, s1);
        if (i + 1 < steps) step(i + 1, s1, s0);
      }
    };
    if (wide) {
      if (stream)
        wide_tile(std::true_type());
      else
        wide_tile(std::false_type());
    } else {
      // Every wave by itself, 32 keys a step: K's buffer takes the next block's as soon as the scores have been worked out, V's as
      // soon as the output has, so that copies are in flight all the time and no two waves wait for each other.
      constexpr int STEP = 128, PER = 512 / STEP;
      const int steps = (end - begin + STEP - 1) / STEP;
      const char *kl = s_kv + wave * 64 * ROW_BYTES, *vl = kl + 32 * ROW_BYTES;
      const uint32_t k_to = lds_address(kl), v_to = lds_address(vl);
      auto rows_of = [&](int i) __attribute__((always_inline)) { return groups(at, (i % PER) * 16 + 4 * wave, std::integral_constant<int, 4>()); };
      auto copy_k = [&](const Groups<4>& g) __attribute__((always_inline)) {
        if (stream)
          copy_groups<true, true>(kb, g, pitch, lc, k_to);
        else
          copy_groups<true, false>(kb, g, pitch, lc, k_to);
      };
      auto copy_v = [&](const Groups<4>& g) __attribute__((always_inline)) {
        if (stream)
          copy_groups<false, true>(vb, g, pitch, lc, v_to);
        else
          copy_groups<false, false>(vb, g, pitch, lc, v_to);
      };
      Groups<4> rows = rows_of(0);
      copy_k(rows);
      copy_v(rows);
      for (int i = 0; i < steps; ++i) {
        const int k0 = begin + i * STEP + 32 * wave, k1 = k0 + 31;
        const bool live = k0 <= wave_hi && k1 >= wave_lo, more = i + 1 < steps;
        f32x16 s[1];
        copies_but<8>();  // K is there (behind it: V's eight copies)
        if (live) s[0] = scores_of<DT>(kl, q);
        lds_read();
        if (more) {
          if ((i + 1) % PER == 0) {
            at = stretch((i + 1) / PER, next);
            next = ask((i + 1) / PER + 1);
          }
          rows = rows_of(i + 1);
          copy_k(rows);
        }
        u32x4 w[2];
        if (live) {
          // (a split ends on a block or with the tile's last key, so what a row sees of a block is in its interval)
          if (SCALED) adjust<CAP, BIAS, 1>(p, s, k0, row, slope_log2);
          if (k0 < all_lo || k1 > all_hi) {
            rarely();
            hide<1>(s, k0, row);
          }
          const float base = new_maximum<SCALED>(p, largest<1>(s), st);
          weigh<DT, SCALED, 1>(p, s, base, w, st);
        }
        if (more)
          copies_but<8>();  // V is there (behind it: the next K's eight)
        else
          copies_done();
        if (live) add_values<DT, 1>(vl, w, st);
        lds_read();
        if (more) copy_v(rows);
      }
    }
  }
  st.l = across_halves(st.l, [](float a, float b) { return a + b; });
  st.lx = across_halves(st.lx, [](float a, float b) { return a + b; });

  const bool one = p.parts == 1 || !cut, none = !one && begin >= end;  // (a split without keys has weight 0: its sum says so)
  const int half = lane >> 5;
  auto put_sums = [&](int64_t at, float m, float l, float lx) __attribute__((always_inline)) {
    if (!one)
      reinterpret_cast<PartSums*>(p.part_ml)[at * p.parts + part0 + split] = PartSums{m, l, lx};
    else if (p.lse)
      p.lse[at] = lx == 0.0f ? -__builtin_inff() : (m + __builtin_log2f(lx)) * LN2;
  };
  auto put = [&](int64_t at, int ch, f32x4 o, float inv) __attribute__((always_inline)) {
    if (one)
      *reinterpret_cast<uint2*>(p.out + at * ABSB_HEAD_DIM + ch) = uint2{pack2<DT>(o[0] * inv, o[1] * inv), pack2<DT>(o[2] * inv, o[3] * inv)};
    else
      *reinterpret_cast<f32x4*>(p.part_o + (at * p.parts + part0 + split) * ABSB_HEAD_DIM + ch) = o;
  };
  if (wide) {
    if (!valid) return;
    const int64_t at = (int64_t)row.row * p.Hq + row.head;
    const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
    if (half == 0) put_sums(at, st.m, st.l, st.lx);
    if (none) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)  // channels 32 i + 8 j + 4 half + 0 .. 3
        put(at, 32 * i + 8 * j + 4 * half, f32x4{st.o[i][4 * j], st.o[i][4 * j + 1], st.o[i][4 * j + 2], st.o[i][4 * j + 3]}, inv);
    return;
  }
  // The waves of a narrow tile have keys of their own: their states become one, eight threads a row.
  __syncthreads();
  float* s_o = reinterpret_cast<float*>(s_kv);  // [wave][row][channel], rows NARROW_PITCH apart
  if (valid) {
    const int col = lane & 31;
    if (half == 0) {
      s_ml[wave][0][col] = st.m;
      s_ml[wave][1][col] = st.l;
      s_ml[wave][2][col] = st.lx;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(s_o + (wave * 32 + col) * NARROW_PITCH + 32 * i + 8 * j + 4 * half) =
            f32x4{st.o[i][4 * j], st.o[i][4 * j + 1], st.o[i][4 * j + 2], st.o[i][4 * j + 3]};
  }
  __syncthreads();
  const int r = (int)threadIdx.x >> 3, c = (int)threadIdx.x & 7;
  if (r >= t.pairs) return;
  const PairOf pair = pair_of_tile(p, t, r);
  const int64_t at = (int64_t)(t.r0 + pair.tok) * p.Hq + kv_head * p.G + pair.g;
  float m = -__builtin_inff(), l = 0.0f, lx = 0.0f, w[ATT_WAVES];
#pragma unroll
  for (int x = 0; x < ATT_WAVES; ++x) m = fmaxf(m, s_ml[x][0][r]);
  const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
  for (int x = 0; x < ATT_WAVES; ++x) {
    w[x] = exp2_fast(s_ml[x][0][r] - base);
    l = __builtin_fmaf(s_ml[x][1][r], w[x], l);
    lx = __builtin_fmaf(s_ml[x][2][r], w[x], lx);
  }
  if (c == 0) put_sums(at, m, l, lx);
  if (none) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int ch = 32 * j + 4 * c;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < ATT_WAVES; ++x) o += *reinterpret_cast<const f32x4*>(s_o + (x * 32 + r) * NARROW_PITCH + ch) * w[x];
    put(at, ch, o, inv);
  }
}

__device__ __forceinline__ float wave_sum(float x) {
  x = row16_sum(x);
  return bitcast<float>(__builtin_amdgcn_readlane(bitcast<int>(x), 0)) + bitcast<float>(__builtin_amdgcn_readlane(bitcast<int>(x), 16)) +
         bitcast<float>(__builtin_amdgcn_readlane(bitcast<int>(x), 32)) + bitcast<float>(__builtin_amdgcn_readlane(bitcast<int>(x), 48));
}

// The parts of a (row, query head), a wave each: half a wave a part, a lane four channels.  TAIL: of the first `n` tile slots only, a
// wave a row of a tile; else of the first `n` pairs.
template <int DT, bool TAIL>
__global__ __launch_bounds__(256) void attend_merge_kernel(AttendParams p, int64_t n) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
  int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (TAIL) {
    const int log2_tile = p.own.log2_tile, i = (int)(at & ((1 << log2_tile) - 1));
    const uint32_t unit = (uint32_t)(at >> log2_tile);
    const int64_t slot = unit / (uint32_t)p.Hkv;
    const Owner own = owner_of(p.own.owners, slot, p.G, log2_tile, p.seq_lens, [&](int o) { return p.row_off[o]; });
    const uint32_t pair = ((uint32_t)(slot - own.slot0) << log2_tile) + (uint32_t)i;
    if (pair >= (uint32_t)(own.r1 - own.r0) * (uint32_t)p.G) return;
    at = (int64_t)(own.r0 + (int)(pair / (uint32_t)p.G)) * p.Hq + (int)(unit % (uint32_t)p.Hkv) * p.G + (int)(pair % (uint32_t)p.G);
  }
  for (; TAIL || at < n; at += (int64_t)gridDim.x * 4) {
    const PartSums* sums = reinterpret_cast<const PartSums*>(p.part_ml) + at * p.parts;
    const float* o = p.part_o + at * p.parts * ABSB_HEAD_DIM + 4 * (lane & 31);
    constexpr int TRIP = 16;  // parts fetched at once
    float M = -__builtin_inff(), L = 0.0f, Lx = 0.0f;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = 0; i0 < p.parts; i0 += 64) {
      PartSums mine = {-__builtin_inff(), 0.0f, 0.0f};
      if (i0 + lane < p.parts) mine = sums[i0 + lane];
      if (mine.l == 0.0f) mine.m = -__builtin_inff();  // (a NaN stays one)
      const float top = fmaxf(M, wave_max_f32(mine.m)), base = top == -__builtin_inff() ? 0.0f : top;
      const float a = exp2_fast(M - base), w = exp2_fast(mine.m - base);
      M = top;
      L = __builtin_fmaf(L, a, mine.l * w);  // (a lane's own parts)
      Lx = __builtin_fmaf(Lx, a, mine.lx * w);
      x *= a;
      const int n = min(64, p.parts - i0);
      for (int i = 0; i < n; i += TRIP) {
        f32x4 v[TRIP / 2];
#pragma unroll
        for (int j = 0; j < TRIP / 2; ++j)
          v[j] = *reinterpret_cast<const f32x4*>(o + (int64_t)(i0 + min(i + 2 * j + half, n - 1)) * ABSB_HEAD_DIM);
#pragma unroll
        for (int j = 0; j < TRIP / 2; ++j) {
          const float wi = __shfl(w, min(i + 2 * j + half, 63));
          if (i + 2 * j + half < n && wi != 0.0f) x += v[j] * wi;  // (an output of weight 0 may never have been written)
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = across_halves(x[j], [](float a, float b) { return a + b; });
    L = wave_sum(L);
    Lx = wave_sum(Lx);
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    if (half == 0)
      *reinterpret_cast<uint2*>(p.out + at * ABSB_HEAD_DIM + 4 * lane) = uint2{pack2<DT>(x[0] * inv, x[1] * inv), pack2<DT>(x[2] * inv, x[3] * inv)};
    if (p.lse && lane == 0) p.lse[at] = Lx == 0.0f ? -__builtin_inff() : (M + __builtin_log2f(Lx)) * LN2;
    if (TAIL) return;
  }
}

template <int DT, int CAP, bool BIAS>
static void launch_parts(const AttendParams& p, int64_t rows, hipStream_t stream) {
  const int64_t own_units = (p.own.whole + (p.own.slots - p.own.whole) * p.own.splits) * p.Hkv;
  hipLaunchKernelGGL((attend_kernel<DT, CAP, BIAS>), dim3((unsigned)(p.shared_units + own_units)), dim3(ATT_THREADS), 0, stream, p);
  if (p.parts > 1 && p.own.whole) {
    const int64_t slots = p.own.slots - p.own.whole;
    hipLaunchKernelGGL((attend_merge_kernel<DT, true>), dim3((unsigned)((slots * p.Hkv << p.own.log2_tile) / 4)), dim3(256), 0, stream, p, slots);
  } else if (p.parts > 1) {
    const int64_t pairs = rows * p.Hq;
    const unsigned grid = (unsigned)std::min<int64_t>((pairs + 3) / 4, MAX_WGS);
    hipLaunchKernelGGL((attend_merge_kernel<DT, false>), dim3(grid), dim3(256), 0, stream, p, pairs);
  }
}
template <int DT, int CAP>
static void launch_capped(const AttendParams& p, int64_t rows, hipStream_t stream) {
  if (p.slopes)
    launch_parts<DT, CAP, true>(p, rows, stream);
  else
    launch_parts<DT, CAP, false>(p, rows, stream);
}
template <int DT>
static void launch_typed(const AttendParams& p, const AttendPlan& plan, float softcap, hipStream_t stream) {
  if (softcap == 0.0f)
    launch_capped<DT, CAP_NONE>(p, plan.rows, stream);
  else if (softcap <= 64.0f)  // (small scores are then off by 64 * 2^-22 = 2^-16 at most)
    launch_capped<DT, CAP_PLAIN>(p, plan.rows, stream);
  else
    launch_capped<DT, CAP_WIDE>(p, plan.rows, stream);
}

int launch_attend(const AttendParams& p, const AttendPlan& plan, int dtype, float softcap, hipStream_t stream) {
  if (dtype == ABSB_F16)
    launch_typed<ABSB_F16>(p, plan, softcap, stream);
  else
    launch_typed<ABSB_BF16>(p, plan, softcap, stream);
  return check_launch();
}

}  // namespace absb
