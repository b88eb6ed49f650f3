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
constexpr int MAP_THREADS = 1024;

struct MapSums {
  int32_t rows, take, give;  // of the requests before a point
};

__global__ __launch_bounds__(MAP_THREADS) void map_rows_kernel(MapParams p) {
  __shared__ int32_t s_rows[MAP_THREADS + 1], s_take[MAP_THREADS + 1], s_give[MAP_THREADS + 1];
  __shared__ int32_t s_before[MAP_THREADS], s_had[MAP_THREADS], s_need[MAP_THREADS];
  __shared__ int32_t s_wave[3][MAP_THREADS / 64], s_short;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lP = p.log2_page, P = 1 << lP;

  int before = 0, after = 0;
  auto read = [&](int b) {
    before = b < p.batch ? max(p.before[b], 0) : 0;
    after = b < p.batch ? max(p.after[b], 0) : 0;
  };
  auto pages_of = [&](int len) { return (int)(((int64_t)len + P - 1) >> lP); };
  // Prefix sums over the MAP_THREADS requests from b0 on, into s_*[0 .. MAP_THREADS]; the requests' own values beside them.
  auto scan = [&](int b0) {
    read(b0 + tid);
    const int had = pages_of(before), need = pages_of(after);
    const uint32_t v[3] = {(uint32_t)max(after - before, 0), (uint32_t)max(need - had, 0), (uint32_t)max(had - need, 0)};
    uint32_t in[3];
    __syncthreads();  // what the last chunk left has been read
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      uint32_t total;
      in[k] = wave_incl_scan_u32(v[k], &total);
      if (lane == 0) s_wave[k][wave] = (int32_t)total;
    }
    s_before[tid] = before;
    s_had[tid] = had;
    s_need[tid] = need;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k)
      for (int w = 0; w < wave; ++w) in[k] += (uint32_t)s_wave[k][w];
    s_rows[tid + 1] = (int32_t)in[0];
    s_take[tid + 1] = (int32_t)in[1];
    s_give[tid + 1] = (int32_t)in[2];
    if (tid == 0) s_rows[0] = s_take[0] = s_give[0] = 0;
    __syncthreads();
  };
  // Largest i in [0, MAP_THREADS) with s[i] <= x (s[0] = 0 <= x < s[MAP_THREADS]): the request that x falls to.
  auto owner = [&](const int32_t* s, int x) {
    int lo = 0;
#pragma unroll
    for (int step = MAP_THREADS / 2; step > 0; step >>= 1)
      if (s[lo + step] <= x) lo += step;
    return lo;
  };

  // ---- the sums of the whole batch, and whether every page can be had
  const bool one_chunk = p.batch <= MAP_THREADS;
  MapSums all = {0, 0, 0};
  int too_long = 0;
  for (int b0 = 0; b0 < p.batch; b0 += MAP_THREADS) {
    scan(b0);
    if (p.ring) too_long += max(0, s_need[tid] - max(p.pt_stride, s_had[tid]));  // pages that its table row has no place for
    all.rows += s_rows[MAP_THREADS];
    all.take += s_take[MAP_THREADS];
    all.give += s_give[MAP_THREADS];
  }
  int64_t head = 0, tail = 0, missing = 0;
  if (p.ring) {
    head = p.cursors[0];
    tail = p.cursors[1];
    if (tid == 0) s_short = 0;
    __syncthreads();
    if (too_long) atomicAdd(&s_short, too_long);
    __syncthreads();
    missing = max((int64_t)0, (int64_t)all.take - (tail - head)) + s_short;
  }
  const bool fine = missing == 0;

  // ---- this work-group's share of the rows, the fresh pages and the pages given back
  const int nwg = gridDim.x, wg = blockIdx.x;
  auto share = [&](int64_t n, int* from, int* to) {
    const int64_t each = (n + nwg - 1) / nwg;
    *from = (int)min(n, wg * each);
    *to = (int)min(n, (wg + 1) * each);
  };
  int r_from, r_to, t_from, t_to, g_from, g_to;
  share(min(all.rows, p.max_rows), &r_from, &r_to);
  share(p.ring && fine ? all.take : 0, &t_from, &t_to);
  share(p.ring && fine ? all.give : 0, &g_from, &g_to);
  MapSums base = {0, 0, 0};
  for (int b0 = 0; b0 < p.batch; b0 += MAP_THREADS) {
    if (!one_chunk) scan(b0);  // (else it is still there)
    const int nb = min(MAP_THREADS, p.batch - b0);
    if (wg == 0 && tid < nb) p.row_off[b0 + tid] = base.rows + s_rows[tid];
    const int r_end = min(r_to, base.rows + s_rows[MAP_THREADS]);
    for (int r = max(r_from, base.rows) + tid; r < r_end; r += MAP_THREADS) {
      const int i = owner(s_rows, r - base.rows), pos = s_before[i] + (r - base.rows - s_rows[i]), page = pos >> lP;
      int64_t slot = -1;
      const bool fresh = p.ring && page >= s_had[i];
      if (fine && (fresh || page < p.pt_stride)) {
        const int32_t phys = fresh
                                 ? p.ring[(head + base.take + s_take[i] + page - s_had[i]) % p.capacity]
                                 : p.page_table[(int64_t)(b0 + i) * p.pt_stride + page];
        slot = ((int64_t)phys << lP) + (pos & (P - 1));
      }
      p.row_pos[r] = pos;
      p.row_slot[r] = slot;
    }
    const int t_end = min(t_to, base.take + s_take[MAP_THREADS]);
    for (int t = max(t_from, base.take) + tid; t < t_end; t += MAP_THREADS) {
      const int i = owner(s_take, t - base.take), page = s_had[i] + (t - base.take - s_take[i]);
      p.page_table[(int64_t)(b0 + i) * p.pt_stride + page] = p.ring[(head + t) % p.capacity];
    }
    const int g_end = min(g_to, base.give + s_give[MAP_THREADS]);
    for (int t = max(g_from, base.give) + tid; t < g_end; t += MAP_THREADS) {
      const int i = owner(s_give, t - base.give), page = s_need[i] + (t - base.give - s_give[i]);
      if (page < p.pt_stride) p.ring[(tail + t) % p.capacity] = p.page_table[(int64_t)(b0 + i) * p.pt_stride + page];
    }
    base.rows += s_rows[MAP_THREADS];
    base.take += s_take[MAP_THREADS];
    base.give += s_give[MAP_THREADS];
  }
  if (wg == 0 && tid == 0) p.row_off[p.batch] = all.rows;
  int f_from, f_to;  // rows behind the last one
  share(max(0, p.max_rows - all.rows), &f_from, &f_to);
  for (int r = all.rows + f_from + tid; r < all.rows + f_to; r += MAP_THREADS) {
    p.row_pos[r] = 0;
    p.row_slot[r] = -1;
  }
  if (!p.ring) return;
  __syncthreads();  // (the cursors have been read by all of the work-group long since)
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
  const int64_t items = (int64_t)p.max_rows + p.batch;
  const int64_t wgs = items <= 2 * MAP_THREADS ? 1 : items / MAP_THREADS;
  const int grid = (int)(wgs < 256 ? wgs : 256);
  hipLaunchKernelGGL(map_rows_kernel, dim3(grid), dim3(MAP_THREADS), 0, stream, p);
  return check_launch();
}

// ------------------------------------------------------------------ rotary positions and the cache write
//
// Pair (x, y) of a token at position p turns by p * f:  (x cos - y sin, x sin + y cos).  The angle is taken in turns, as a
// 64-bit fraction F = f / 2 pi mod 1, so that p * F mod 2^64 is the exact product whatever the position: in binary32 an angle
// of a million radians is off by 0.03.  Its upper 32 bits, as a number in [-1/2, 1/2), go to the hardware's sine and cosine
// of turns (off by at most 1.3e-7 over that range, where a 16-bit result is off by 2^-12 at best).
//
// Bound by memory: (Hq + 2 Hkv) rows of 256 bytes in and out a token.  A lane holds 16-byte pieces (of both halves of a pair's
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

// Where head h of a row is read from and written to (queries, then keys, then values).
struct HeadIo {
  const uint16_t* src;
  uint16_t* dst;  // null: nowhere
  bool turn;
};
__device__ __forceinline__ HeadIo head_io(const RotateParams& p, int row, int h, int64_t slot) {
  HeadIo io;
  if (h < p.nq) {
    io.src = p.q + row * p.q_stride + h * ABSB_HEAD_DIM;
    io.dst = p.q_out + ((int64_t)row * p.nq + h) * ABSB_HEAD_DIM;
    io.turn = true;
    return io;
  }
  h -= p.nq;
  const bool key = h < p.nkv;
  if (!key) h -= p.nkv;
  io.src = (key ? p.k + row * p.k_stride : p.v + row * p.v_stride) + h * ABSB_HEAD_DIM;
  uint16_t* cache = key ? p.k_cache : p.v_cache;
  io.dst = slot < 0 ? nullptr
                    : cache + (slot >> p.log2_page) * p.s_page + (int64_t)h * p.s_head + (slot & ((1 << p.log2_page) - 1)) * p.s_tok;
  io.turn = key;
  return io;
}

// Halves of whole pieces (rot_dim a multiple of 16), or neighbours (of 8): LANES lanes a head.
template <int DT, bool PAIRS, int LANES>
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
    const HeadIo io = head_io(p, row, h, slot);
    if (!io.dst || !used) continue;
    u32x4 a = *reinterpret_cast<const u32x4*>(io.src + ca), b = {0u, 0u, 0u, 0u};
    const bool two = !PAIRS && turns;
    if (two) b = *reinterpret_cast<const u32x4*>(io.src + cb);
    if (io.turn && turns) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (PAIRS) {
          const float x = Elem<DT>::lo(a[w]), y = Elem<DT>::hi(a[w]);
          const float u = x * cs[w % N] - y * sn[w % N], v = x * sn[w % N] + y * cs[w % N];
          a[w] = (uint32_t)Elem<DT>::narrow(u) | ((uint32_t)Elem<DT>::narrow(v) << 16);
        } else {
          const float x0 = Elem<DT>::lo(a[w]), y0 = Elem<DT>::lo(b[w]), x1 = Elem<DT>::hi(a[w]), y1 = Elem<DT>::hi(b[w]);
          const int i = 2 * w % N, j = (2 * w + 1) % N;
          a[w] = (uint32_t)Elem<DT>::narrow(x0 * cs[i] - y0 * sn[i]) | ((uint32_t)Elem<DT>::narrow(x1 * cs[j] - y1 * sn[j]) << 16);
          b[w] = (uint32_t)Elem<DT>::narrow(x0 * sn[i] + y0 * cs[i]) | ((uint32_t)Elem<DT>::narrow(x1 * sn[j] + y1 * cs[j]) << 16);
        }
      }
    }
    *reinterpret_cast<u32x4*>(io.dst + ca) = a;
    if (two) *reinterpret_cast<u32x4*>(io.dst + cb) = b;
  }
}

// Any even rot_dim: a lane takes pair `lane` of a head (two channels apart by any distance) and, behind the pairs, channels
// that pass two by two.
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
    const HeadIo io = head_io(p, row, h, slot);
    if (!io.dst) continue;
    uint16_t a = io.src[ca], b = io.src[cb];
    if (io.turn && turns) {
      const float x = Elem<DT>::widen(a), y = Elem<DT>::widen(b);
      a = Elem<DT>::narrow(x * cs - y * sn);
      b = Elem<DT>::narrow(x * sn + y * cs);
    }
    io.dst[ca] = a;
    io.dst[cb] = b;
  }
}

template <int DT>
static void launch_rotate_typed(const RotateParams& p, dim3 grid, int lanes, hipStream_t stream) {
  if (lanes == 64)
    hipLaunchKernelGGL((rotate_any_kernel<DT>), grid, dim3(256), 0, stream, p);
  else if (!p.halves)
    hipLaunchKernelGGL((rotate_kernel<DT, true, 16>), grid, dim3(256), 0, stream, p);
  else if (lanes == 8)
    hipLaunchKernelGGL((rotate_kernel<DT, false, 8>), grid, dim3(256), 0, stream, p);
  else
    hipLaunchKernelGGL((rotate_kernel<DT, false, 16>), grid, dim3(256), 0, stream, p);
}

int launch_rotate(RotateParams p, int dtype, hipStream_t stream) {
  // lanes a head: the pieces that pass beside the pairs of pieces that turn, up to a power of two (8 when all channels turn)
  const int lanes = p.rot % (p.halves ? 16 : 8) ? 64 : p.halves && p.rot == ABSB_HEAD_DIM ? 8 : 16;
  const int heads = p.nq + 2 * p.nkv, at_once = 64 / lanes;
  // few tokens: a wave takes as many heads as it holds at once; many: a token
  p.parts = (heads + at_once - 1) / at_once;
  if ((int64_t)p.n_rows * p.parts > 8192) p.parts = 1;
  p.heads_per_part = ((heads + p.parts - 1) / p.parts + at_once - 1) / at_once * at_once;
  const int64_t grid = ((int64_t)p.n_rows * p.parts + 3) / 4;
  if (dtype == ABSB_F16)
    launch_rotate_typed<ABSB_F16>(p, dim3((unsigned)grid), lanes, stream);
  else
    launch_rotate_typed<ABSB_BF16>(p, dim3((unsigned)grid), lanes, stream);
  return check_launch();
}

}  // namespace absb
