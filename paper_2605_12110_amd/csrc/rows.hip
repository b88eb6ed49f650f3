// The rows of a step: where new tokens go in the paged cache (absb_map_rows), and their rotary positions with the cache
// write (absb_rotate_store).
#include "common.h"
#include "rows.h"

namespace absb {

// ------------------------------------------------------------------ rows, slots and page tables
//
// With n_b = max(0, after_b - before_b), had_b = ceil(before_b / P), need_b = ceil(after_b / P): row off_b + i is token
// before_b + i, and request b's fresh page j (had_b <= j < need_b) is entry head + T_b + j - had_b of the ring, T the prefix
// sums of max(0, need - had).  Three prefix sums over the requests decide everything.
//
// One launch: every work-group sums over all requests by itself (8 bytes a request, from the L2) and then does its share of the
// rows, of the fresh pages and of the pages given back, so that none waits for another.  Nothing written here is
// read here: a row in a fresh page takes it from the ring, not from the table.  The cursors change at the end of the call only,
// written by the work-group that finishes last, since until then others may be reading them.
//
// Bound by latency: lengths in, page table or ring in, rows out, and two barriers between.  As few threads as cover the batch: a
// barrier costs by its waves (64 requests, a token each: 3.4, 3.6 and 4.8 us with 256, 512 and 1024 threads), a second round over
// the batch more (300: 7.2, 5.2, 6.3; 600: 9.2, 8.8, 6.3; 2000: 17.5, 12.8, 12.7).
struct MapSums {
  int32_t rows, take, give;  // of the requests before a point
};

template <int T>
__global__ __launch_bounds__(T) void map_rows_kernel(MapParams p) {
  constexpr int WAVES = T / 64;
  __shared__ int32_t s_rows[T + 1], s_take[T + 1], s_give[T + 1];
  __shared__ int32_t s_before[T], s_had[T], s_need[T];
  __shared__ int32_t s_wave[4][WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lP = p.log2_page, P = 1 << lP;
  const bool ring = p.ring != nullptr;
  const uint32_t cap = (uint32_t)p.capacity;
  int64_t head = 0, tail = 0;
  if (ring) {
    head = p.cursors[0];
    tail = p.cursors[1];
  }

  // Prefix sums over the T requests from b0 on, into s_*[0 .. T]; the requests' own values beside them.  Returns how many pages
  // to take or to give back the tables have no place for.
  auto scan = [&](int b0, bool first) __attribute__((always_inline)) {
    const int b = b0 + tid;
    const int before = b < p.batch ? max(p.before[b], 0) : 0, after = b < p.batch ? max(p.after[b], 0) : 0;
    const int had = (int)(((int64_t)before + P - 1) >> lP), need = (int)(((int64_t)after + P - 1) >> lP);
    const uint32_t v[4] = {(uint32_t)max(after - before, 0), (uint32_t)max(need - had, 0), (uint32_t)max(had - need, 0),
                           ring ? (uint32_t)max(0, max(need, had) - max(p.pt_stride, min(need, had))) : 0u};
    uint32_t in[4];
    if (!first) __syncthreads();  // what the last chunk left has been read
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t total;
      in[k] = wave_incl_scan_u32(v[k], &total);
      if (lane == 0) s_wave[k][wave] = (int32_t)total;
    }
    s_before[tid] = before;
    s_had[tid] = had;
    s_need[tid] = need;
    __syncthreads();
    int short_of = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
#pragma unroll
      for (int k = 0; k < 3; ++k) in[k] += w < wave ? (uint32_t)s_wave[k][w] : 0u;
      short_of += s_wave[3][w];
    }
    s_rows[tid + 1] = (int32_t)in[0];
    s_take[tid + 1] = (int32_t)in[1];
    s_give[tid + 1] = (int32_t)in[2];
    if (tid == 0) s_rows[0] = s_take[0] = s_give[0] = 0;
    __syncthreads();
    return short_of;
  };
  // Largest i in [0, T) with s[i] <= x (s[0] = 0 <= x < s[T]): the request that x falls to.
  auto owner = [&](const int32_t* s, int x) __attribute__((always_inline)) {
    int lo = 0;
#pragma unroll
    for (int step = T / 2; step > 0; step >>= 1)
      if (s[lo + step] <= x) lo += step;
    return lo;
  };

  // ---- the sums of the whole batch, and whether every page can be had
  const bool one_chunk = p.batch <= T;
  MapSums all = {0, 0, 0};
  int64_t missing = 0;
  for (int b0 = 0; b0 < p.batch; b0 += T) {
    missing += scan(b0, b0 == 0);
    all.rows += s_rows[T];
    all.take += s_take[T];
    all.give += s_give[T];
  }
  if (ring) missing += max((int64_t)0, (int64_t)all.take - (tail - head));
  const bool fine = missing == 0;
  // entry `from` + i of the ring: no division but this one
  auto first_place = [&](int64_t from) { return (uint64_t)from >> 32 ? (uint32_t)((uint64_t)from % cap) : (uint32_t)from % cap; };
  const uint32_t head0 = ring ? first_place(head) : 0, tail0 = ring ? first_place(tail) : 0;
  auto place = [&](uint32_t first, int i) __attribute__((always_inline)) {
    const uint64_t at = (uint64_t)first + (uint32_t)i;
    return at < cap ? (uint32_t)at : at - cap < cap ? (uint32_t)(at - cap) : (uint32_t)(at % cap);
  };

  // ---- this work-group's share of the rows, the fresh pages and the pages given back
  const int nwg = gridDim.x, wg = blockIdx.x;
  struct Share {
    int from, to;
  };
  auto share = [&](int n) __attribute__((always_inline)) {
    if (nwg == 1) return Share{0, n};
    const uint32_t each = ((uint32_t)n + nwg - 1) / (uint32_t)nwg;
    return Share{(int)min((uint64_t)n, (uint64_t)wg * each), (int)min((uint64_t)n, (uint64_t)(wg + 1) * each)};
  };
  const Share r = share(min(all.rows, p.max_rows)), take = share(ring && fine ? all.take : 0), give = share(ring && fine ? all.give : 0);
  MapSums base = {0, 0, 0};
  for (int b0 = 0; b0 < p.batch; b0 += T) {
    if (!one_chunk) scan(b0, false);  // (else it is still there)
    if (wg == 0 && tid < p.batch - b0) p.row_off[b0 + tid] = base.rows + s_rows[tid];
    const int r_end = min(r.to, base.rows + s_rows[T]);
    for (int x = max(r.from, base.rows) + tid; x < r_end; x += T) {
      const int i = owner(s_rows, x - base.rows), pos = s_before[i] + (x - base.rows - s_rows[i]), page = pos >> lP;
      const bool fresh = ring && page >= s_had[i];
      int64_t slot = -1;
      if (fine && (fresh || page < p.pt_stride)) {
        const int32_t* at = fresh ? p.ring + place(head0, base.take + s_take[i] + page - s_had[i])
                                  : p.page_table + ((int64_t)(b0 + i) * p.pt_stride + page);
        slot = ((int64_t)*at << lP) + (pos & (P - 1));
      }
      p.row_pos[x] = pos;
      p.row_slot[x] = slot;
    }
    const int t_end = min(take.to, base.take + s_take[T]);
    for (int x = max(take.from, base.take) + tid; x < t_end; x += T) {
      const int i = owner(s_take, x - base.take), page = s_had[i] + (x - base.take - s_take[i]);
      p.page_table[(int64_t)(b0 + i) * p.pt_stride + page] = p.ring[place(head0, x)];
    }
    // Four pages a thread at once: the host does not know how many come back, and a round trip serves four (256 requests of 5000
    // tokens in pages of 8, all finished: 105 us -> 56 with twice the work-groups, 143 before both).
    constexpr int AT_ONCE = 4;
    const int g_end = min(give.to, base.give + s_give[T]);
    for (int x0 = max(give.from, base.give) + tid; x0 < g_end; x0 += AT_ONCE * T) {
      int32_t phys[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int x = min(x0 + j * T, g_end - 1), i = owner(s_give, x - base.give), page = s_need[i] + (x - base.give - s_give[i]);
        phys[j] = p.page_table[(int64_t)(b0 + i) * p.pt_stride + page];
      }
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
        if (x0 + j * T < g_end) p.ring[place(tail0, x0 + j * T)] = phys[j];
    }
    base.rows += s_rows[T];
    base.take += s_take[T];
    base.give += s_give[T];
  }
  if (wg == 0 && tid == 0) p.row_off[p.batch] = all.rows;
  const Share fill = share(max(0, p.max_rows - all.rows));  // rows behind the last one
  for (int x = fill.from + tid; x < fill.to; x += T) {
    p.row_pos[all.rows + x] = 0;
    p.row_slot[all.rows + x] = -1;
  }
  if (!ring) return;
  // The cursors: by the work-group that comes last, since all the others have read them by then.
  __syncthreads();
  if (tid == 0) {
    unsigned long long* done = reinterpret_cast<unsigned long long*>(p.cursors_out + 3);
    if (nwg == 1 || __hip_atomic_fetch_add(done, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned long long)nwg - 1) {
      p.cursors_out[0] = head + (fine ? all.take : 0);
      p.cursors_out[1] = tail + (fine ? all.give : 0);
      p.cursors_out[2] = missing;
      __hip_atomic_store(done, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
}

int launch_map_rows(const MapParams& p, hipStream_t stream) {
  // Two rows a thread, and with a ring a work-group for every 64 requests, whose pages the host does not know; at most 192: the
  // last one, who sets the cursors, hears from all the others one after the other (a step of 512 requests and 302803
  // rows 10.0 us with 192, 10.3 with 256, 10.6 with 96; of 151570 rows 8.65 with 148, 8.6 with 96, 8.9 with 74).
  const int threads = p.batch <= 256 ? 256 : p.batch <= 512 ? 512 : 1024;
  const int by_rows = p.max_rows <= 2 * threads ? 1 : p.max_rows / (2 * threads), by_pages = p.ring ? p.batch / 64 : 1;
  const int wgs = by_rows > by_pages ? by_rows : by_pages;
  const int grid = wgs < 1 ? 1 : wgs < 192 ? wgs : 192;
  if (threads == 256)
    hipLaunchKernelGGL((map_rows_kernel<256>), dim3(grid), dim3(256), 0, stream, p);
  else if (threads == 512)
    hipLaunchKernelGGL((map_rows_kernel<512>), dim3(grid), dim3(512), 0, stream, p);
  else
    hipLaunchKernelGGL((map_rows_kernel<1024>), dim3(grid), dim3(1024), 0, stream, p);
  return check_launch();
}

// ------------------------------------------------------------------ rotary positions and the cache write
//
// Pair (x, y) of a token at position p turns by p * f:  (x cos - y sin, x sin + y cos).  The angle is taken in turns, as a
// 64-bit fraction F = f / 2 pi mod 1, so that p * F mod 2^64 is the exact product whatever the position: in binary32 an angle
// of a million radians is off by 0.03.  Its upper 32 bits, as a number in [-1/2, 1/2), go, rounded to the 24 of
// binary32 (2^-26 turns at most), to the hardware's sine and cosine of turns (off by at most 1.3e-7 over that range, where a 16-bit
// result is off by 2^-12 at best).
//
// Bound by memory: (Hq + 2 Hkv) rows of 256 bytes in and out a token (8192 tokens of 48 heads 39 us, 32 K 140 us, 5.2 and 5.65 TB/s;
// 16 tokens 3.9 us, a chain of round trips).  A lane holds 16-byte pieces (of both halves of a pair's
// channels), LANES of them a head; a wave works on one token and a stretch of its heads, so that the sines are worked out once for
// several heads.
__device__ __forceinline__ uint64_t turns_of(double f) {
  double t = f * 0.15915494309189533577;  // 1 / 2 pi
  t -= floor(t);                          // [0, 1], exact for |t| < 2^52
  const double hi = floor(t * 4294967296.0);
  const double lo = (t * 4294967296.0 - hi) * 4294967296.0;
  return ((uint64_t)(uint32_t)(uint64_t)hi << 32) + (uint64_t)(uint32_t)lo;
}
__device__ __forceinline__ void sin_cos(uint64_t F, int32_t pos, float amplitude, float* s, float* c) {
  const int32_t frac = (int32_t)(uint32_t)((F * (uint64_t)(int64_t)pos) >> 32);
  const float t = (float)frac * 0x1p-32f;
  *s = __builtin_amdgcn_sinf(t) * amplitude;
  *c = __builtin_amdgcn_cosf(t) * amplitude;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Where head h of a row is read from and written to (queries, then keys, then values; null: nowhere).
__device__ __forceinline__ const uint16_t* head_src(const RotateParams& p, int row, int h) {
  if (h < p.nq) return p.q + row * p.q_stride + h * ABSB_HEAD_DIM;
  h -= p.nq;
  return h < p.nkv ? p.k + row * p.k_stride + h * ABSB_HEAD_DIM : p.v + row * p.v_stride + (h - p.nkv) * ABSB_HEAD_DIM;
}
__device__ __forceinline__ uint16_t* head_dst(const RotateParams& p, int row, int h, int64_t slot) {
  if (h < p.nq) return p.q_out + ((int64_t)row * p.nq + h) * ABSB_HEAD_DIM;
  if (slot < 0) return nullptr;
  h -= p.nq;
  const bool key = h < p.nkv;
  return (key ? p.k_cache : p.v_cache) + (slot >> p.log2_page) * p.s_page + (int64_t)(key ? h : h - p.nkv) * p.s_head +
         (slot & ((1 << p.log2_page) - 1)) * p.s_tok;
}
// Two values rounded to the K/V type, side by side.
template <int DT>
__device__ __forceinline__ uint32_t pair_of(float a, float b) {
  if (DT == ABSB_F16) return bitcast<uint32_t>(half2_t{(_Float16)a, (_Float16)b});
  return bitcast<uint32_t>(bf16x2_t{(__bf16)a, (__bf16)b});
}

// Halves of whole pieces (rot_dim a multiple of 16), or neighbours (of 8): LANES lanes a head.
// PAST: what passes the caches by: nothing, reads, or writes too.
enum : int { PAST_NONE = 0, PAST_READS = 1, PAST_ALL = 2 };
template <int DT, bool PAIRS, int LANES, int PAST>
__global__ __launch_bounds__(256) void rotate_kernel(RotateParams p) {
  constexpr int HEADS = 64 / LANES;  // a wave does at a time
  const int task = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = task / p.parts, part = task - row * p.parts;
  if (row >= p.n_rows) return;
  const int piece = lane % LANES, h0 = part * p.heads_per_part + lane / LANES;
  const int h_end = min(p.nq + 2 * p.nkv, (part + 1) * p.heads_per_part);
  // this lane's pieces of a head: `a`, and for halves its partner `b` (of channels that pass: the lane's one piece is `a`)
  const int turned = PAIRS ? p.rot / 8 : p.rot / 16;  // lanes that turn pairs
  const bool turns = piece < turned;
  const int ca = (PAIRS || turns ? piece : piece + turned) * 8, cb = (piece + turned) * 8;
  const bool used = ca < ABSB_HEAD_DIM;
  // A head's pieces are asked for ahead of what is done with them: the first ahead of the sines, the next ahead of the one before.
  u32x4 a = {0u, 0u, 0u, 0u}, b = a;
  const bool two = !PAIRS && turns;
  auto fetch = [&](int h) __attribute__((always_inline)) {
    if (h >= h_end || !used) return;
    const uint16_t* src = head_src(p, row, h);
    auto piece_at = [&](int c) {
      const u32x4* at = reinterpret_cast<const u32x4*>(src + c);
      return PAST == PAST_NONE ? *at : __builtin_nontemporal_load(at);
    };
    a = piece_at(ca);
    if (two) b = piece_at(cb);
  };
  fetch(h0);
  const int pos = p.pos[row];
  const int64_t slot = p.slot ? p.slot[row] : -1;
  constexpr int N = PAIRS ? 4 : 8;  // pairs of a lane
  float sn[N], cs[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sn[i] = 0.0f;
    cs[i] = 1.0f;
    if (turns) sin_cos(turns_of(p.freq[piece * N + i]), pos, p.amplitude, &sn[i], &cs[i]);
  }
  for (int h = h0; h < h_end; h += HEADS) {
    u32x4 x = a, y = b;
    fetch(h + HEADS);
    uint16_t* dst = head_dst(p, row, h, slot);
    if (!dst || !used) continue;
    if (turns && h < p.nq + p.nkv) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (PAIRS) {
          const float u = Elem<DT>::lo(x[w]), v = Elem<DT>::hi(x[w]);
          x[w] = pair_of<DT>(u * cs[w % N] - v * sn[w % N], u * sn[w % N] + v * cs[w % N]);
        } else {
          const float x0 = Elem<DT>::lo(x[w]), y0 = Elem<DT>::lo(y[w]), x1 = Elem<DT>::hi(x[w]), y1 = Elem<DT>::hi(y[w]);
          const int i = 2 * w % N, j = (2 * w + 1) % N;
          x[w] = pair_of<DT>(x0 * cs[i] - y0 * sn[i], x1 * cs[j] - y1 * sn[j]);
          y[w] = pair_of<DT>(x0 * sn[i] + y0 * cs[i], x1 * sn[j] + y1 * cs[j]);
        }
      }
    }
    auto put = [&](int c, u32x4 v) {
      u32x4* at = reinterpret_cast<u32x4*>(dst + c);
      if (PAST == PAST_ALL)
        __builtin_nontemporal_store(v, at);
      else
        *at = v;
    };
    put(ca, x);
    if (two) put(cb, y);
  }
}

// Any even rot_dim: a lane takes pair `lane` of a head (two channels apart by any distance) and, behind the pairs, channels
// that pass two by two.  Two bytes a lane, a head after the other: 8192 tokens of 48 heads 66 us, 3.1 TB/s.
template <int DT>
__global__ __launch_bounds__(256) void rotate_any_kernel(RotateParams p) {
  const int task = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = task / p.parts, part = task - row * p.parts;
  if (row >= p.n_rows) return;
  const int h_end = min(p.nq + 2 * p.nkv, (part + 1) * p.heads_per_part);
  const int half = p.rot / 2;
  const bool turns = lane < half;
  const int ca = turns && p.halves ? lane : 2 * lane, cb = turns && p.halves ? lane + half : 2 * lane + 1;
  const int64_t slot = p.slot ? p.slot[row] : -1;
  float sn = 0.0f, cs = 1.0f;
  if (turns) sin_cos(turns_of(p.freq[lane]), p.pos[row], p.amplitude, &sn, &cs);
  for (int h = part * p.heads_per_part; h < h_end; ++h) {
    uint16_t* dst = head_dst(p, row, h, slot);
    if (!dst) continue;
    const uint16_t* src = head_src(p, row, h);
    uint16_t a = src[ca], b = src[cb];
    if (turns && h < p.nq + p.nkv) {
      const float x = Elem<DT>::widen(a), y = Elem<DT>::widen(b);
      a = Elem<DT>::narrow(x * cs - y * sn);
      b = Elem<DT>::narrow(x * sn + y * cs);
    }
    dst[ca] = a;
    dst[cb] = b;
  }
}

template <int DT, int PAST>
static void launch_rotate_typed(const RotateParams& p, dim3 grid, int lanes, hipStream_t stream) {
  if (lanes == 64)
    hipLaunchKernelGGL((rotate_any_kernel<DT>), grid, dim3(256), 0, stream, p);
  else if (!p.halves)
    hipLaunchKernelGGL((rotate_kernel<DT, true, 16, PAST>), grid, dim3(256), 0, stream, p);
  else if (lanes == 8)
    hipLaunchKernelGGL((rotate_kernel<DT, false, 8, PAST>), grid, dim3(256), 0, stream, p);
  else
    hipLaunchKernelGGL((rotate_kernel<DT, false, 16, PAST>), grid, dim3(256), 0, stream, p);
}
template <int DT>
static void launch_rotate_sized(const RotateParams& p, dim3 grid, int lanes, hipStream_t stream) {
  // Rows that no cache keeps for the next reader pass it by: 100 MB read and as much written (8192 tokens of 48 heads) 45.6 us, with
  // reads past the caches 38.4, with writes too 40.4; 75 MB each 29.7, 29.5, 30.4; 200 MB 85, 84, 77; 50 MB 18.4, 21.0, 21.5.
  const double mb = (double)p.n_rows * (p.nq + 2 * p.nkv) * ABSB_HEAD_DIM * 2 / (1 << 20);
  if (mb < 64)
    launch_rotate_typed<DT, PAST_NONE>(p, grid, lanes, stream);
  else if (mb < 144)
    launch_rotate_typed<DT, PAST_READS>(p, grid, lanes, stream);
  else
    launch_rotate_typed<DT, PAST_ALL>(p, grid, lanes, stream);
}

int launch_rotate(RotateParams p, int dtype, hipStream_t stream) {
  // lanes a head: the pieces that pass beside the pairs of pieces that turn, up to a power of two (8 when all channels turn)
  const int lanes = p.rot % (p.halves ? 16 : 8) ? 64 : p.halves && p.rot == ABSB_HEAD_DIM ? 8 : 16;
  const int heads = p.nq + 2 * p.nkv, at_once = 64 / lanes;
  // few tokens: a wave takes as many heads as it holds at once; many: a token (48 heads, 64 tokens: 3.5 us, and 5.6 with a token a
  // wave; 700: both 6.6; 2048: 15.9 and 9.9)
  p.parts = (heads + at_once - 1) / at_once;
  if ((int64_t)p.n_rows * p.parts > 8192) p.parts = 1;
  p.heads_per_part = ((heads + p.parts - 1) / p.parts + at_once - 1) / at_once * at_once;
  const int64_t grid = ((int64_t)p.n_rows * p.parts + 3) / 4;
  if (dtype == ABSB_F16)
    launch_rotate_sized<ABSB_F16>(p, dim3((unsigned)grid), lanes, stream);
  else
    launch_rotate_sized<ABSB_BF16>(p, dim3((unsigned)grid), lanes, stream);
  return check_launch();
}

}  // namespace absb
